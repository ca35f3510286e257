// Which pages of a cache a query has to read: bounds of every page's keys, scores from them, the highest ones.
//
// Bounds.  For a page and key head the smallest and the largest of its tokens' keys, value by value.  Only pages with new tokens are gone through;
// memory bounds it (their keys).  A workgroup takes a page and a head, its wavefronts some of the rows, a lane 4 - 16 bytes of a row.  A cache in 8 bits
// has bounds in bfloat16, rounded outwards where its scales are no powers of two.  (24 streams with 300 new tokens each, 8 heads of 128 in 8 bits: 6 us; with
// sums over rows in LDS 21.)
//
// Scores.  sum_d max(q_d lo_d, q_d hi_d) is no less than q.k for any key k of the page; a page's score is the largest of its key head's query heads.  Sums
// are in float64 and rounded to float32 once: products of float32 values are exact there, and a sum is off by dim * 2^-53 of its terms' sizes at most, so that their
// order shows only in scores that lie as near to where float32's rounding changes, or whose terms all but cancel.  The order is fixed, whatever pages and heads a call has:
// the matrix cores' 4 x 4 x 4 products in four blocks, 16 pages and 4 query heads at once, of hi with the positive parts of q and of lo with the negative
// ones, each summed by itself (vector instructions took 7 us where these take 3: they convert every value for every query head).  Memory bounds it: 2 * dim values a page and key head.
//
// Choice.  The workgroup that comes last of those that have made a (sequence, key head)'s scores finds the lowest score that is taken by counting digits
// (radix selection, ten bits a pass between the lowest and the highest score), then lists the pages in order.  Sequences whose pages are all taken
// need no scores.  3 126 pages of 8 key heads with 4 query heads each: 13 us, of which 3 are the way to the bounds, 3.6 the
// scores, 2 until all workgroups have arrived, 4.5 the choice: steps that follow from each other.  (A launch of its own for the choice, by 1 024 threads: 16 us.)
#include <type_traits>

#include "cb_tokens.h"

namespace cb {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int pages_of(const Cache& c, int seq)
{
    return (clamp_length(c.lengths[seq], c.capacity) + (1 << c.page_shift) - 1) >> c.page_shift;
}

// ---------------------------------------------------------------- bounds
constexpr int BOUND_THREADS = 256, BOUND_WAVES = BOUND_THREADS / 64;

// To bfloat16, up or down; what is not a number stays so.
__device__ __forceinline__ uint16_t outwards(float f, bool up)
{
    const uint32_t b = __float_as_uint(f);
    if (f != f) return 0x7FC0;
    const bool away = (b & 0xFFFFu) != 0 && up == ((b >> 31) == 0);      // from zero
    return (uint16_t)((b >> 16) + (away ? 1 : 0));
}

// The sequence that unit u belongs to and its number there, if every sequence has n(sequence) of them; -1: there are fewer.  The same for all
// lanes of a wavefront.
struct Found { int seq, unit; };
template <typename N> __device__ __forceinline__ Found find_unit(const Cache& c, int u, N n)
{
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < c.seqs; s0 += 64) {
        const int sum = wave_scan(s0 + lane < c.seqs ? n(s0 + lane) : 0);
        const unsigned long long past = __ballot(sum > u);
        if (past) {
            const int at = __builtin_ctzll(past);
            return Found{s0 + at, u - (at > 0 ? __builtin_amdgcn_readlane(sum, at - 1) : 0)};
        }
        u -= __builtin_amdgcn_readlane(sum, 63);
    }
    return Found{-1, 0};
}

// Values of W bytes of a row.
template <typename KT, int BYTES> __device__ __forceinline__ void widen_row(const uint32_t (&w)[BYTES / 4], float (&f)[BYTES / sizeof(KT)])
{
#pragma unroll
    for (int i = 0; i < BYTES / 4; ++i) {
        if constexpr (sizeof(KT) == 4) f[i] = __uint_as_float(w[i]);
        else if constexpr (sizeof(KT) == 2) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        } else {
            f[4 * i] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 0);
            f[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 1);
            f[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 2);
            f[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 3);
        }
    }
}

// BYTES of a row a lane, as few as leave a row 64 lanes.
template <typename KT, int BYTES>
__global__ __launch_bounds__(BOUND_THREADS) void bound_kernel(const int32_t* since, const Cache c)
{
    constexpr int N = BYTES / sizeof(KT), AHEAD = BYTES == 16 ? 4 : 8;      // rows that are on their way at once
    typedef uint32_t word_t __attribute__((ext_vector_type(BYTES / 4)));
    __shared__ float s_part[BOUND_WAVES][2][256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), per_row = c.dim / N;
    int log = 0;                                               // lanes of a row
    while (1 << log < per_row) ++log;
    const int sub = lane & ((1 << log) - 1), at_once = 64 >> log, row0 = wave * at_once + (lane >> log), step = BOUND_WAVES * at_once;
    auto first_page = [&](int s) {
        const int pages = pages_of(c, s), from = since ? clamp_length(since[s], c.capacity) >> c.page_shift : 0;
        return from < pages ? from : pages;
    };
    auto units = [&](int s) { return (pages_of(c, s) - first_page(s)) * c.heads; };
    for (int u = blockIdx.x;; u += gridDim.x) {
        const Found now = find_unit(c, u, units);
        if (now.seq < 0) return;
        const int at = now.unit / c.heads, h = now.unit - at * c.heads, p = first_page(now.seq) + at;
        const int page = c.table[(long)now.seq * c.max_pages + p], left = clamp_length(c.lengths[now.seq], c.capacity) - (p << c.page_shift);
        if ((unsigned)page < (unsigned)c.n_pages) {
            const int rows = left < 1 << c.page_shift ? left : 1 << c.page_shift;
            const long head = (long)page * c.heads + h;
            const KT* src = (const KT*)c.k + (head << c.page_shift) * c.dim + sub * N;
            const float* scale = c.k_scale + (head << (c.page_shift - 4));
            float lo[N], hi[N];
#pragma unroll
            for (int i = 0; i < N; ++i) { lo[i] = __builtin_inff(); hi[i] = -__builtin_inff(); }
            const int end = sub < per_row ? rows : 0;
            for (int r0 = row0; r0 < end; r0 += AHEAD * step) {
                word_t w[AHEAD];
                float y[AHEAD];
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) {
                    // (behind the last row the first one again)
                    const int r = r0 + a * step < end ? r0 + a * step : r0;
                    w[a] = *reinterpret_cast<const word_t*>(src + (long)r * c.dim);
                    if constexpr (sizeof(KT) == 1) y[a] = scale[r >> 4];
                }
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) {
                    uint32_t words[BYTES / 4];
                    __builtin_memcpy(words, &w[a], BYTES);
                    float x[N];
                    widen_row<KT, BYTES>(words, x);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        if constexpr (sizeof(KT) == 1) x[i] *= y[a];
                        lo[i] = __builtin_elementwise_minimum(lo[i], x[i]);      // (what is not a number stays)
                        hi[i] = __builtin_elementwise_maximum(hi[i], x[i]);
                    }
                }
            }
            for (int k = log; k < 6; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    lo[i] = __builtin_elementwise_minimum(lo[i], __shfl_xor(lo[i], 1 << k));
                    hi[i] = __builtin_elementwise_maximum(hi[i], __shfl_xor(hi[i], 1 << k));
                }
            if (lane < per_row)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    s_part[wave][0][sub * N + i] = lo[i];
                    s_part[wave][1][sub * N + i] = hi[i];
                }
            __syncthreads();
            for (int d = tid; d < 2 * c.dim; d += BOUND_THREADS) {
                const bool up = d >= c.dim;
                const int x = up ? d - c.dim : d;
                float y = s_part[0][up][x];
#pragma unroll
                for (int k = 1; k < BOUND_WAVES; ++k)
                    y = up ? __builtin_elementwise_maximum(y, s_part[k][1][x]) : __builtin_elementwise_minimum(y, s_part[k][0][x]);
                const long to = head * 2 * c.dim + d;
                if constexpr (sizeof(KT) == 1) ((uint16_t*)c.bounds)[to] = outwards(y, up);
                else if constexpr (sizeof(KT) == 2) narrow(y, ((uint16_t*)c.bounds)[to]);
                else ((float*)c.bounds)[to] = y;
            }
            __syncthreads();
        }
    }
}

// ---------------------------------------------------------------- scores and choice
constexpr int THREADS = 512, WAVES = THREADS / 64, DIGIT = 10, BINS = 1 << DIGIT;
constexpr int ROW = 16, PAGES = WAVES * ROW;      // pages that a wavefront scores at a time, and a workgroup
constexpr int HEADS = 4;                         // query heads at a time
constexpr int ROUNDS = 2, SPAN = 4 * THREADS * ROUNDS;      // ranks that a thread holds at once, in fours; all threads
constexpr uint32_t ALWAYS = 0xFFFFFFFFu;         // above every score's rank
static_assert(BINS == 2 * THREADS, "two bins a thread");

struct ChooseArgs {
    ChooseJob j;
    Cache c;
    int group;                           // query heads of a key head
    int* counters;                       // of (sequence, key head)
    uint32_t* ranks;                     // of (sequence, key head)
    long pitch;
};

__device__ __forceinline__ void put_rank(uint32_t* at, uint32_t r) { __hip_atomic_store(at, r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// Four of them, as other compute units have written them.
__device__ __forceinline__ u32x4 get_ranks(__amdgpu_buffer_rsrc_t ranks, int at)
{
    constexpr int AGENT = 16;
    return __builtin_amdgcn_raw_buffer_load_b128(ranks, at * 4, 0, AGENT);
}

// Sum over the threads before this one.
__device__ __forceinline__ int sum_before(int v, int* s_part)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sum = wave_scan(v);
    if (lane == 63) s_part[wave] = sum;
    __syncthreads();
    const int parts = wave_scan(lane < WAVES ? s_part[lane] : 0);
    return sum - v + (wave > 0 ? __builtin_amdgcn_readlane(parts, wave - 1) : 0);
}

// Units of work, dealt to the workgroups in turn: a block of PAGES of a (sequence, key head), the only one of a sequence whose pages are all taken.
// WHOLE: all blocks of one, where there are more pairs than counters.
template <typename BT, typename T, bool WHOLE>
__global__ __launch_bounds__(THREADS) void choose_kernel(const ChooseArgs a)
{
    constexpr int N = 16 / sizeof(BT), AHEAD = 4;      // values of 16 bytes; pieces of both bounds that are on their way at once
    // positive and negative parts of q, of a piece's values one behind the other, pieces a bank's width apart (without it four lanes meet in one bank)
    __shared__ __align__(16) double2 s_q[256 / N][N + 1][HEADS];
    __shared__ __align__(16) int hist[BINS];
    __shared__ int s_part[2][WAVES], s_count[2][ROUNDS][WAVES], s_pick[3], s_last;
    __shared__ uint32_t s_low, s_high;
    __shared__ __align__(16) uint32_t s_rank[PAGES];
    const Cache& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), budget = a.j.budget, pieces = c.dim / N;
    auto blocks_of = [&](int s) {
        const int pages = pages_of(c, s);
        return WHOLE || pages <= budget ? 1 : (pages + PAGES - 1) / PAGES;
    };
    for (int u = blockIdx.x;; u += gridDim.x) {
        const Found f = find_unit(c, u, [&](int s) { return blocks_of(s) * c.heads; });
        if (f.seq < 0) return;
        const int seq = f.seq, blocks = blocks_of(seq), h = f.unit / blocks, first = f.unit - h * blocks, n = pages_of(c, seq);
        const long pair = (long)seq * c.heads + h;
        int32_t* chosen = a.j.chosen + pair * budget;
        if (n <= budget) {
            for (int i = tid; i < budget; i += THREADS) chosen[i] = i < n ? i : -1;
            if (tid == 0) a.j.count[pair] = n;
            continue;
        }
        uint32_t* ranks = a.ranks + pair * a.pitch;
        const bool alone = n <= PAGES;               // ranks do not leave the workgroup
        for (int block = first; block < (WHOLE ? (n + PAGES - 1) / PAGES : first + 1); ++block) {
            // lane: page l % 16 and every fourth piece of 16 bytes of its bounds, from l / 16 on
            const int quad = lane >> 4, p = block * PAGES + wave * ROW + (lane & 15);
            int page = -1;
            if (p < n) page = c.table[(long)seq * c.max_pages + p];
            const bool there = (unsigned)page < (unsigned)c.n_pages;
            const BT* bounds = (const BT*)c.bounds + (there ? ((long)page * c.heads + h) * 2 * c.dim : 0);
            // what is in this lane in the end: page 4 * (l / 4 % 4) + l / 16 for query head l % 4
            const int at = (lane >> 2 & 3) * 4 + quad;
            float best = -__builtin_inff();
            for (int g0 = 0; g0 < a.group; g0 += HEADS) {
                double up = 0.0, down = 0.0;
#pragma unroll 1
                for (int i0 = 0; i0 < pieces; i0 += 4 * AHEAD) {
                    u32x4 lo[AHEAD], hi[AHEAD];
#pragma unroll
                    for (int x = 0; x < AHEAD; ++x) {
                        const int i = i0 + 4 * x + quad;
                        lo[x] = hi[x] = u32x4(0);
                        if (there && i < pieces) {
                            lo[x] = *reinterpret_cast<const u32x4*>(bounds + i * N);
                            hi[x] = *reinterpret_cast<const u32x4*>(bounds + c.dim + i * N);
                        }
                    }
                    if (i0 == 0) {
                        __syncthreads();         // (the parts of q that were there have been read)
                        for (int i = tid; i < HEADS * 256; i += THREADS) {
                            const int g = i >> 8, d = i & 255, head = h * a.group + (g0 + g < a.group ? g0 + g : g0);
                            double q = 0.0;
                            if (d < c.dim) q = (double)widen(((const T*)a.j.q.data)[(long)seq * a.j.q.token + (long)head * a.j.q.head + d]);
                            s_q[d / N][d % N][g] = q != q ? make_double2(q, q) : make_double2(q > 0.0 ? q : 0.0, q < 0.0 ? q : 0.0);
                        }
                        __syncthreads();
                    }
#pragma unroll
                    for (int x = 0; x < AHEAD; ++x) {
                        if (i0 + 4 * x >= pieces) continue;
                        // (all of a piece's parts of q first: one at a time they would come a trip to LDS apart)
                        const double2* q = &s_q[i0 + 4 * x + quad][0][lane & 3];
                        double2 part[N];
#pragma unroll
                        for (int e = 0; e < N; ++e) part[e] = q[e * HEADS];
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            auto value = [&](const u32x4& w) {
                                if constexpr (sizeof(BT) == 4) return (double)__uint_as_float(w[e]);
                                else return (double)__uint_as_float(e % 2 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
                            };
                            up = __builtin_amdgcn_mfma_f64_4x4x4f64(value(hi[x]), part[e].x, up, 0, 0, 0);
                            down = __builtin_amdgcn_mfma_f64_4x4x4f64(value(lo[x]), part[e].y, down, 0, 0, 0);
                        }
                    }
                }
                float score = (float)(up + down);
                score = score != score ? __builtin_inff() : score;                    // (what is not a number rules nothing out)
                auto from = [](float x, auto step) { return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), step.value, 0xf, 0xf, true)); };
                score = fmaxf(score, from(score, std::integral_constant<int, 0xB1>()));      // quad_perm 1 0 3 2
                score = fmaxf(score, from(score, std::integral_constant<int, 0x4E>()));      // quad_perm 2 3 0 1
                best = fmaxf(best, score);
            }
            // ranks in the scores' order; above all of them the pages that are always taken, below pages without a number, which hold no token
            const unsigned long long any = __ballot(there);
            const int of = block * PAGES + wave * ROW + at;
            if (of < n && (lane & 3) == 0) {
                const uint32_t b = __float_as_uint((any >> at & 1 ? best : -__builtin_inff()) + 0.0f);
                s_rank[wave * ROW + at] = of < a.j.first || of >= n - a.j.recent ? ALWAYS : (b & 0x80000000u ? ~b : b | 0x80000000u);
            }
            __syncthreads();
            // (a wavefront stores them all: whoever waits for its stores has waited for all)
            if (!alone && wave == 0)
#pragma unroll
                for (int i = lane; i < PAGES; i += 64)
                    if (block * PAGES + i < n) put_rank(ranks + block * PAGES + i, s_rank[i]);
            if (WHOLE) __syncthreads();
        }
        if (!alone) {
            if (tid < 64) {
                __builtin_amdgcn_s_waitcnt(0x0F70);      // vmcnt(0): this wavefront's stores are where every compute unit sees them
                if (tid == 0) {
                    int* counter = a.counters + pair;
                    s_last = WHOLE || __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == blocks - 1;
                    if (s_last && !WHOLE) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
            }
            __syncthreads();
            const bool last = s_last;
            __syncthreads();
            if (!last) continue;
        }
        if (tid == 0) { s_low = 0xFFFFFFFFu; s_high = 0; }

        // Ranks are gone through SPAN at a time, those of pages 4 * (tid + THREADS * i) .. in round i; up to SPAN of them stay in registers.  0: no page.
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(ranks, 0, (int)(a.pitch * 4), 0x00027000);
        u32x4 r[ROUNDS];
        auto load = [&](int base) {
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i) {
                const int at = base + 4 * (tid + THREADS * i);
                if (!alone) r[i] = get_ranks(from, at);            // (zero behind the array)
                else if (at < PAGES) r[i] = *reinterpret_cast<const u32x4*>(s_rank + at);
                else r[i] = u32x4(0);
            }
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x) r[i][x] = base + 4 * (tid + THREADS * i) + x < n ? r[i][x] : 0u;
        };
        auto each = [&](auto f) {                    // all of them
#pragma unroll 1
            for (int base = 0; base < n; base += SPAN) {
                if (n > SPAN) load(base);
#pragma unroll
                for (int i = 0; i < ROUNDS; ++i) {
                    if (base + 4 * THREADS * i >= n) continue;
#pragma unroll
                    for (int x = 0; x < 4; ++x) f(r[i][x]);
                }
            }
        };
        load(0);
        uint32_t low = 0xFFFFFFFFu, high = 0;
        each([&](uint32_t k) {
            low = min(low, k - 1u);
            high = max(high, k == ALWAYS ? 0u : k);
        });
        low = ~wave_max_unsigned(~low);
        high = wave_max_unsigned(high);
        __syncthreads();
        if (lane == 0) { atomicMin(&s_low, low); atomicMax(&s_high, high); }
        *reinterpret_cast<int2*>(hist + 2 * tid) = make_int2(0, 0);
        __syncthreads();
        low = s_low + 1u;
        high = s_high;
        // `want` of those that rank low .. high are taken, all that rank above are.  (Those that are always taken are fewer than the budget, or
        // as many: then none of the others is.)
        int want = budget - (a.j.first + a.j.recent);
        bool found = want == 0;
        if (found) low = high = ALWAYS - 1;
        // (ten bits a pass: four at most, whatever the ranks are)
        for (int pass = 0; pass < 4 && !found; ++pass) {
            const int turn = pass & 1;
            const int bits = 32 - __builtin_clz((high - low) | 1u), shift = bits > DIGIT ? bits - DIGIT : 0;
            each([&](uint32_t k) {
                if (k >= low && k <= high) atomicAdd(&hist[(k - low) >> shift], 1);
            });
            __syncthreads();
            // from the highest digit down, two digits a thread
            const int bin = BINS - 2 * (tid + 1);
            const int2 here = *reinterpret_cast<const int2*>(hist + bin);
            const int above = sum_before(here.x + here.y, s_part[turn]);
            *reinterpret_cast<int2*>(hist + bin) = make_int2(0, 0);
            if (above < want && above + here.y >= want) { s_pick[0] = bin + 1; s_pick[1] = above; s_pick[2] = here.y; }
            else if (above + here.y < want && above + here.y + here.x >= want) { s_pick[0] = bin; s_pick[1] = above + here.y; s_pick[2] = here.x; }
            __syncthreads();
            low += (uint32_t)s_pick[0] << shift;
            const uint32_t end = low + ((1u << shift) - 1u);
            high = end < high ? end : high;
            want -= s_pick[1];
            found = shift == 0 || want == s_pick[2];
        }
        // the pages in order: in every round those of the threads before, and those of the rounds before
        int before = 0, ties = 0;                    // of the spans before
#pragma unroll 1
        for (int base = 0, turn = 0; base < n; base += SPAN, turn ^= 1) {
            if (n > SPAN) load(base);
            // (both in one: sure ones above bit 16, equal ones below; up to 256 in a wavefront)
            int sums[ROUNDS];
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i) {
                if (base + 4 * THREADS * i >= n) continue;
                int own = 0;
#pragma unroll
                for (int x = 0; x < 4; ++x) own += (r[i][x] > high ? 1 << 16 : 0) + (r[i][x] >= low && r[i][x] <= high ? 1 : 0);
                sums[i] = wave_scan(own) - own;
                if (lane == 63) s_count[turn][i][wave] = sums[i] + own;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i) {
                if (base + 4 * THREADS * i >= n) continue;
                // (sums of all wavefronts do not fit 16 bits: one after the other)
                const int of = lane < WAVES ? s_count[turn][i][lane] : 0, of_sure = wave_scan(of >> 16), of_equal = wave_scan(of & 0xFFFF);
                int sure = before + (sums[i] >> 16) + (wave > 0 ? __builtin_amdgcn_readlane(of_sure, wave - 1) : 0);
                int equal = ties + (sums[i] & 0xFFFF) + (wave > 0 ? __builtin_amdgcn_readlane(of_equal, wave - 1) : 0);
                before += __builtin_amdgcn_readlane(of_sure, 63);
                ties += __builtin_amdgcn_readlane(of_equal, 63);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint32_t k = r[i][x];
                    const int p = base + 4 * (tid + THREADS * i) + x;
                    const bool tie = k >= low && k <= high;
                    const int to = sure + (equal < want ? equal : want);
                    if ((k > high || (tie && equal < want)) && to < budget) chosen[to] = p;
                    sure += k > high;
                    equal += tie;
                }
            }
        }
        if (tid == 0) a.j.count[pair] = budget;
        __syncthreads();                             // (LDS is the next unit's)
    }
}

}  // namespace

// (units and pages of all sequences are counted in 32 bits)
bool choose_fits(const Cache& c) { return (unsigned long long)c.seqs * c.heads * c.max_pages < (1ull << 30); }

hipError_t launch_bound(const int32_t* since, const Cache& c, hipStream_t st)
{
    const long most = (long)c.seqs * c.heads * c.max_pages, want = 8L * device_units();
    const dim3 grid((unsigned)(most < want ? most : want)), block(BOUND_THREADS);
    // (a row has 64 lanes at most: 4 bytes each where those reach)
#define CB_BOUND(type, b) hipLaunchKernelGGL((bound_kernel<type, b>), grid, block, 0, st, since, c)
    if (c.e4m3) CB_BOUND(uint8_t, 4);
    else if (c.bf16) {
        if (c.dim <= 128) CB_BOUND(uint16_t, 4);
        else CB_BOUND(uint16_t, 8);
    } else {
        if (c.dim <= 64) CB_BOUND(float, 4);
        else if (c.dim <= 128) CB_BOUND(float, 8);
        else CB_BOUND(float, 16);
    }
#undef CB_BOUND
    return hipGetLastError();
}

hipError_t launch_choose(const ChooseJob& j, const Cache& c, hipStream_t st)
{
    ChooseArgs a;
    a.j = j;
    a.c = c;
    a.group = j.q.heads / c.heads;
    a.counters = reinterpret_cast<int*>(c.scratch) + CHOOSE_COUNTERS;
    a.ranks = reinterpret_cast<uint32_t*>(c.scratch + scratch_plan(c, 0).pages);
    a.pitch = rank_pitch(c);
    // as many workgroups as are at work at once, no more than there can be units
    const long pairs = (long)c.seqs * c.heads, blocks = (c.max_pages + PAGES - 1) / PAGES, want = 2L * device_units();
    const bool whole = pairs > CHOOSE_PAIRS;
    const long most = whole || j.budget >= c.max_pages ? pairs : pairs * blocks;
    const dim3 grid((unsigned)(most < want ? most : want)), block(THREADS);
#define CB_CHOOSE(bounds, values) do { if (whole) hipLaunchKernelGGL((choose_kernel<bounds, values, true>), grid, block, 0, st, a); \
                                       else hipLaunchKernelGGL((choose_kernel<bounds, values, false>), grid, block, 0, st, a); } while (0)
    if (c.e4m3 && !c.bf16) CB_CHOOSE(uint16_t, float);
    else if (c.e4m3 || c.bf16) CB_CHOOSE(uint16_t, uint16_t);
    else CB_CHOOSE(float, float);
#undef CB_CHOOSE
    return hipGetLastError();
}

}  // namespace cb
