// Eviction from a paged cache by accumulated attention weight.
//
// Every (sequence, key head) keeps `budget` of its tokens: the recent ones (time above the newest - window), then those with the
// largest weight.  One workgroup each finds the smallest kept rank by counting the ranks' digits from the highest to the lowest (radix
// selection: no sorting), and lists, in ascending order, the free slots below the budget and the kept tokens above it.
// There are as many of one as of the other; a second launch moves them.  Sources and targets never overlap, so nothing waits
// for anything, and only what has to move moves.
//
// The selection reads weights and times from memory at once, and keeps the ranks in LDS, where the counting's passes find
// them; those of more slots than it holds are made again from memory in every pass.  16 x 8 heads of 17 000 - 25 000 tokens: 28 us, and 88 us for the
// moves (425 MB read and written, 4.8 TB/s).  One sequence with 310 of 2 358 tokens to go: 7.2 us, about 20 steps that follow from each other, and 3.
#include "cb_tokens.h"

namespace cb {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int DIGIT = 10, BINS = 1 << DIGIT;      // bits of a digit; a bin a thread
constexpr int COPIES = 4;                        // of a histogram: lanes that count the same digit do not queue up behind each other
constexpr int STRIDE = 4 * THREADS;              // slots of all threads, four each
constexpr int LDS_RANKS = 30720;
static_assert(BINS == THREADS, "a bin a thread");

struct EvictArgs {
    EvictJob j;
    Cache c;
    int32_t *count, *hole, *mover;       // per (sequence, head): how many, their slots (pitch = capacity)
    int copies;                          // weight or time have to be copied where a token stays
    int room;                            // ranks that LDS holds
};

// In the order of the numbers; what is not a number comes first, and zeros are equal.  Rank 0 is for what is below all others: weights that
// are not a number, the earliest time there is, and the slots up to three behind the last token, which come behind all tokens of rank 0.
__device__ __forceinline__ uint32_t ordered(float f)
{
    if (f != f) return 0u;
    const uint32_t b = __float_as_uint(f + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint32_t ordered(int32_t t) { return (uint32_t)t ^ 0x80000000u; }
constexpr uint32_t RECENT = 0xFFFFFFFFu;         // above every weight's rank

// The sum over the lanes before this one, and over all.
__device__ __forceinline__ int lane_sum_before(int v, int* all)
{
    const int sum = wave_scan(v);
    *all = __builtin_amdgcn_readlane(sum, 63);
    return (int)((uint32_t)sum - (uint32_t)v);
}

// The sum of all wavefronts' entries before this one's.
__device__ __forceinline__ int before_wave(const int* s_part, int wave)
{
    const int lane = threadIdx.x & 63;
    int all;
    return __builtin_amdgcn_readlane(lane_sum_before(lane < WAVES ? s_part[lane] : 0, &all), wave);
}

// ALL_IN_LDS: of every sequence that the cache has room for.  1 024 threads: an
// earlier form took 8.5 us for 8 heads of 2 358 tokens, 9.1 with 512 and 10.3 with 256.
template <bool ALL_IN_LDS>
__global__ __launch_bounds__(THREADS) void select_kernel(const EvictArgs a)
{
    extern __shared__ __align__(16) uint32_t s_rank[];
    __shared__ __align__(16) int hist[2][BINS * COPIES];     // of this digit, and the next one's, empty
    __shared__ int s_part[WAVES], s_equal[WAVES], s_hole[WAVES], s_mover[WAVES];
    __shared__ int s_newest, s_recent, s_pick[3];
    __shared__ uint32_t s_low, s_high;
    const Cache& c = a.c;
    const int seq = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long pair = (long)seq * c.heads + h, at = pair * c.capacity;
    const int len = clamp_length(a.j.lengths_in[seq], c.capacity), budget = a.j.budget;
    const float* weight = a.j.weight_in + at;
    const int32_t* time = a.j.time_in + at;

    if (tid == 0) {
        s_newest = INT32_MIN;
        s_recent = 0;
        s_low = 0xFFFFFFFFu;
        s_high = 0;
    }
    *reinterpret_cast<i32x4*>(hist[0] + 4 * tid) = i32x4{0, 0, 0, 0};
    // Times and weights, four slots a thread (a row ends behind a multiple of 16).  Where others than the cache's own decide, the cache
    // receives them: of free slots too, which the moves write over.
    const bool in_lds = ALL_IN_LDS || len <= a.room;
    int newest = INT32_MIN;
    i32x4 t0 = {0, 0, 0, 0};                                   // times of a thread's first four slots
    // (both as read: then as the ranks want them)
    auto take_over = [&](int i, i32x4& t, f32x4& w) {
        if (a.copies && i < budget) {
            if (i + 4 <= budget && i + 4 <= len) {
                *reinterpret_cast<f32x4*>(c.weight + at + i) = w;
                *reinterpret_cast<i32x4*>(c.time + at + i) = t;
            } else
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (i + x < budget && i + x < len) {
                        c.weight[at + i + x] = w[x];
                        c.time[at + i + x] = t[x];
                    }
        }
        if (i + 4 > len)
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (i + x >= len) {
                    t[x] = INT32_MIN;
                    w[x] = __builtin_nanf("");
                }
    };
#pragma unroll 4
    for (int i = 4 * tid; i < len; i += STRIDE) {
        i32x4 t = *reinterpret_cast<const i32x4*>(time + i);
        f32x4 w = *reinterpret_cast<const f32x4*>(weight + i);
        take_over(i, t, w);
        newest = max(max(newest, max(t[0], t[1])), max(t[2], t[3]));
        if (in_lds) *reinterpret_cast<u32x4*>(s_rank + i) = u32x4{ordered(w[0]), ordered(w[1]), ordered(w[2]), ordered(w[3])};
        if (i < STRIDE) t0 = t;
    }
    if (len <= budget) {
        if (tid == 0) a.count[pair] = 0;
        return;
    }
    newest = wave_max(newest);
    __syncthreads();
    if (lane == 0) atomicMax(&s_newest, newest);
    __syncthreads();
    // times from here on are recent, if any are
    const long earliest = (long)s_newest - a.j.window + 1;
    const int recent_from = earliest < INT32_MIN ? INT32_MIN : (earliest > INT32_MAX ? INT32_MAX : (int)earliest);
    const bool any_recent = a.j.window > 0;
    bool by_time = false;
    auto ranks_of = [&](const i32x4& t, const u32x4& of_weight) {
        u32x4 k;
#pragma unroll
        for (int x = 0; x < 4; ++x) k[x] = by_time ? ordered(t[x]) : (any_recent && t[x] >= recent_from ? RECENT : of_weight[x]);
        return k;
    };
    auto ranks = [&](int i) -> u32x4 {                         // of slots i .. i + 3
        if (in_lds) return *reinterpret_cast<const u32x4*>(s_rank + i);
        const f32x4 w = *reinterpret_cast<const f32x4*>(weight + i);
        u32x4 k = ranks_of(*reinterpret_cast<const i32x4*>(time + i), u32x4{ordered(w[0]), ordered(w[1]), ordered(w[2]), ordered(w[3])});
#pragma unroll
        for (int x = 1; x < 4; ++x) k[x] = i + x < len ? k[x] : 0u;
        return k;
    };

    // All that rank above `least` stay, and the first `left` of those that rank at it.
    int left;
#pragma unroll 1
    for (;;) {
        // how many are recent, and between which ranks the others are (rank 0 left aside)
        int recent = 0, all;
        uint32_t low = 0xFFFFFFFFu, high = 0;
        auto note = [&](const u32x4& k) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const bool out = !by_time && k[x] == RECENT;
                recent += out;
                low = min(low, k[x] - 1u);
                high = out ? high : max(high, k[x]);
            }
        };
        if (in_lds) {
#pragma unroll 1
            for (int i = 4 * tid; i < len; i += STRIDE) {
                i32x4 t = t0;
                if (i >= STRIDE) {
                    t = *reinterpret_cast<const i32x4*>(time + i);
#pragma unroll
                    for (int x = 1; x < 4; ++x) t[x] = i + x < len ? t[x] : INT32_MIN;
                }
                const u32x4 k = ranks_of(t, *reinterpret_cast<const u32x4*>(s_rank + i));
                *reinterpret_cast<u32x4*>(s_rank + i) = k;
                note(k);
            }
        } else
            for (int i = 4 * tid; i < len; i += STRIDE) note(ranks(i));
        low = ~wave_max_unsigned(~low);
        high = wave_max_unsigned(high);
        lane_sum_before(recent, &all);
        if (lane == 0) {
            atomicMin(&s_low, low);
            atomicMax(&s_high, high);
            atomicAdd(&s_recent, all);
        }
        __syncthreads();
        left = by_time ? budget : budget - s_recent;
        if (left > 0) break;
        // there are as many recent tokens as the budget holds: the newest of all are kept
        by_time = true;
        __syncthreads();
        if (tid == 0) { s_low = 0xFFFFFFFFu; s_high = 0; }
        __syncthreads();
    }
    // (there are more others than are left to keep, since there are more tokens than the budget holds)
    const uint32_t low = s_low + 1u, range = s_high - low;     // (none above rank 0: nothing is in a range that begins behind its end)
    bool at_zero = s_high == 0;
    uint32_t least = 0;
    int shift = 32 - __builtin_clz(range | 1) - DIGIT;
#pragma unroll 1
    for (int past = 32, turn = 0; s_high != 0; turn ^= 1) {
        int* counts = hist[turn];
        shift = shift < 0 ? 0 : shift;
        *reinterpret_cast<i32x4*>(hist[turn ^ 1] + 4 * tid) = i32x4{0, 0, 0, 0};
        // (recent tokens are out of range but where the range ends with them: then there are none)
#pragma unroll 2
        for (int i = 4 * tid; i < len; i += STRIDE) {
            const u32x4 r = ranks(i);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t k = r[x] - low;
                if (k <= range && (past == 32 || (k ^ least) >> past == 0))
                    atomicAdd(&counts[((k >> shift) & (BINS - 1)) * COPIES + (lane & (COPIES - 1))], 1);
            }
        }
        __syncthreads();
        // from the highest digit down, a digit a thread
        const int digit = BINS - 1 - tid;
        const i32x4 bin = *reinterpret_cast<const i32x4*>(counts + digit * COPIES);
        const int n = bin[0] + bin[1] + bin[2] + bin[3];
        int all, counted;
        int above = lane_sum_before(n, &all);
        if (lane == 0) s_part[wave] = all;
        __syncthreads();
        above += __builtin_amdgcn_readlane(lane_sum_before(lane < WAVES ? s_part[lane] : 0, &counted), wave);
        if (past == 32 && counted < left) {
            // fewer than are left: all of them stay, and the first of rank 0
            left -= counted;
            at_zero = true;
            break;
        }
        if (above < left && above + n >= left) {
            s_pick[0] = digit;
            s_pick[1] = left - above;
            s_pick[2] = n;
        }
        __syncthreads();
        least |= (uint32_t)s_pick[0] << shift;
        left = s_pick[1];
        if (shift > 0 && left == s_pick[2]) {
            // all of them stay, whatever their lower digits (there are others below: low + least is not zero)
            --least;
            left = 0;
            break;
        }
        if (shift == 0) break;
        past = shift;
        shift -= DIGIT;
    }
    least = at_zero ? 0u : least + low;

    // Which stay, and where the free slots and the tokens that move into them come in their lists.  A wavefront has a stretch of slots, 256 at
    // a time: first all count theirs, then they list them.
    const int last = budget < len ? budget : len, stretch = (len + STRIDE - 1) / STRIDE * 256;
    const int from = wave * stretch < len ? wave * stretch : len, to = from + stretch < len ? from + stretch : len;
    int equal = 0, hole = 0, mover = 0;                        // before this wavefront's, then before the slots that come
    if (left > 0) {
#pragma unroll 1
        for (int i = from + 4 * lane; i < to; i += 256) {
            const u32x4 k = ranks(i);
#pragma unroll
            for (int x = 0; x < 4; ++x) equal += i + x < len && k[x] == least;
        }
        int all;
        lane_sum_before(equal, &all);
        if (lane == 0) s_equal[wave] = all;
        __syncthreads();
        equal = before_wave(s_equal, wave);
    }
#pragma unroll 1
    for (int list = 0; list < 2; ++list) {
        int run = equal;
#pragma unroll 1
        for (int i0 = from; i0 < to; i0 += 256) {
            const int i = i0 + 4 * lane;
            const u32x4 k = i < to ? ranks(i) : u32x4{0, 0, 0, 0};
            uint32_t kept = 0;
#pragma unroll
            for (int x = 0; x < 4; ++x) kept |= (uint32_t)(k[x] > least) << x;
            if (left > 0) {
                int own = 0, all;
#pragma unroll
                for (int x = 0; x < 4; ++x) own += i + x < to && k[x] == least;
                int at_least = run + lane_sum_before(own, &all);
                run += all;
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (i + x < to && k[x] == least) kept |= (uint32_t)(at_least++ < left) << x;
            }
            const uint32_t low4 = i + 4 <= last ? 15u : (i >= last ? 0u : (1u << (last - i)) - 1);
            const uint32_t holes = low4 & ~kept, movers = kept & ~low4;
            if (!list) {
                hole += (int)__popc(holes);
                mover += (int)__popc(movers);
            } else if (__ballot(holes | movers)) {
                int all;                                       // (both counts in one number)
                const int before = lane_sum_before((int)(__popc(holes) | __popc(movers) << 16), &all);
                int h_at = hole + (before & 0xFFFF), m_at = mover + (before >> 16);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if (holes >> x & 1) a.hole[at + h_at++] = i + x;
                    if (movers >> x & 1) a.mover[at + m_at++] = i + x;
                }
                hole += all & 0xFFFF;
                mover += all >> 16;
            }
        }
        if (!list) {
            int holes, movers;
            lane_sum_before(hole, &holes);
            lane_sum_before(mover, &movers);
            if (lane == 0) { s_hole[wave] = holes; s_mover[wave] = movers; }
            __syncthreads();
            hole = before_wave(s_hole, wave);
            mover = before_wave(s_mover, wave);
        }
    }
    if (wave == WAVES - 1 && lane == 0) a.count[pair] = mover;
}

// Moves: 16-byte pieces of keys and values, weight and time; the sequences' lengths.
__global__ __launch_bounds__(256) void move_kernel(const EvictArgs a)
{
    const Cache& c = a.c;
    const int seq = blockIdx.z, h = blockIdx.y;
    const long pair = (long)seq * c.heads + h, at = pair * c.capacity;
    const int n = a.count[pair], pieces = c.dim * (c.bf16 ? 2 : 4) / 16;
    const int32_t* table = c.table + (long)seq * c.max_pages;
    auto row = [&](int slot) -> long {                     // in pieces; -1: no page
        const int page = table[slot >> c.page_shift];
        if ((unsigned)page >= (unsigned)c.n_pages) return -1;
        return ((((long)page * c.heads + h) << c.page_shift) + (slot & ((1 << c.page_shift) - 1))) * pieces;
    };
    u32x4 *k = (u32x4*)c.k, *v = (u32x4*)c.v;
    // a thread's piece p of its rows
    const int at_once = 256 / pieces, r = threadIdx.x / pieces, p = threadIdx.x - r * pieces;
    if (r < at_once)
        for (int m = blockIdx.x * at_once + r; m < n; m += gridDim.x * at_once) {
            const int from = a.mover[at + m], to = a.hole[at + m];
            const long src = row(from), dst = row(to);
            if (src >= 0 && dst >= 0) {
                const u32x4 x = __builtin_nontemporal_load(k + src + p), y = __builtin_nontemporal_load(v + src + p);
                __builtin_nontemporal_store(x, k + dst + p);
                __builtin_nontemporal_store(y, v + dst + p);
            }
            if (p == 0) {
                c.weight[at + to] = a.j.weight_in[at + from];
                c.time[at + to] = a.j.time_in[at + from];
            }
        }
    if (h == 0 && blockIdx.x == 0 && threadIdx.x == 0) {
        const int len = clamp_length(a.j.lengths_in[seq], c.capacity);
        c.lengths[seq] = len < a.j.budget ? len : a.j.budget;
    }
}

}  // namespace

hipError_t launch_evict(const EvictJob& j, const Cache& c, hipStream_t st)
{
    const ScratchPlan plan = scratch_plan(c, 0);
    EvictArgs a;
    a.j = j;
    a.c = c;
    const long pairs = (long)c.seqs * c.heads;
    a.count = reinterpret_cast<int32_t*>(c.scratch + plan.moves);
    a.hole = a.count + pairs;
    a.mover = a.hole + pairs * c.capacity;
    a.copies = j.weight_in != c.weight || j.time_in != c.time;
    a.room = c.capacity < LDS_RANKS ? c.capacity : LDS_RANKS;
    const dim3 grid(c.heads, c.seqs), block(THREADS);
    if (c.capacity <= LDS_RANKS) hipLaunchKernelGGL(select_kernel<true>, grid, block, a.room * 4, st, a);
    else hipLaunchKernelGGL(select_kernel<false>, grid, block, a.room * 4, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // workgroups of the moves: 64 for each compute unit (128 heads of 3 000 tokens each: 102 us with 8, 91 with 64), no more than the most there
    // can be to move
    const long most = ((long)(c.capacity - j.budget < j.budget ? c.capacity - j.budget : j.budget) * (c.dim * (c.bf16 ? 2 : 4) / 16) + 255) / 256;
    long per = (64L * device_units() + pairs - 1) / pairs;
    per = per > most ? most : per;
    hipLaunchKernelGGL(move_kernel, dim3((unsigned)(per < 1 ? 1 : per), c.heads, c.seqs), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace cb
