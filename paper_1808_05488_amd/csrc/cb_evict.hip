// Eviction from a paged cache by accumulated attention weight.
//
// Every (sequence, key head) keeps `budget` of its tokens: the recent ones (time above the newest - window), then those with the
// largest weight.  One workgroup each finds the smallest kept rank by counting the ranks' bytes from the highest to the lowest (radix
// selection: no sorting), and lists, in ascending order, the free slots below the budget and the kept tokens above it.
// There are as many of one as of the other; a second launch moves them.  Sources and targets never overlap, so nothing waits
// for anything, and only what has to move moves.
#include "cb_tokens.h"

namespace cb {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64, COPIES = 32;

struct EvictArgs {
    EvictJob j;
    Cache c;
    int32_t *count, *hole, *mover;       // per (sequence, head): how many, their slots (pitch = capacity)
    int copies;                          // weight or time have to be copied where a token stays
};

// In the order of the numbers; what is not a number comes first, and zeros are equal.
__device__ __forceinline__ uint32_t ordered(float f)
{
    if (f != f) return 0u;
    const uint32_t b = __float_as_uint(f + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint32_t ordered(int32_t t) { return (uint32_t)t ^ 0x80000000u; }

// What decides about a slot.
struct Ranks {
    const float* weight;
    const int32_t* time;
    long newest;          // - window: times above it are recent
    bool by_time;         // there are as many recent tokens as the budget holds: the newest of them
    __device__ bool recent(int i) const { return (long)time[i] > newest; }
    // rank among the tokens that compete; in: does it compete
    __device__ uint32_t rank(int i, bool* in) const
    {
        if (by_time) { *in = true; return ordered(time[i]); }
        *in = !recent(i);
        return ordered(weight[i]);
    }
};

__device__ int block_sum(int v, int* s_part)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
    __syncthreads();
    int sum = 0;
    for (int w = 0; w < WAVES; ++w) sum += s_part[w];
    return sum;
}

__global__ __launch_bounds__(THREADS) void select_kernel(const EvictArgs a)
{
    __shared__ int hist[256 * COPIES];
    __shared__ int s_bin[256];
    __shared__ int s_part[WAVES], s_hole[WAVES], s_mover[WAVES];
    __shared__ int s_pick, s_left;
    const Cache& c = a.c;
    const int seq = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long pair = (long)seq * c.heads + h, at = pair * c.capacity;
    const int len = clamp_length(a.j.lengths_in[seq], c.capacity), budget = a.j.budget;
    Ranks r{a.j.weight_in + at, a.j.time_in + at, 0, false};

    if (len <= budget) {
        if (tid == 0) a.count[pair] = 0;
        if (a.copies)
            for (int i = tid; i < len; i += THREADS) {
                c.weight[at + i] = r.weight[i];
                c.time[at + i] = r.time[i];
            }
        return;
    }

    int newest = INT32_MIN;
    for (int i = tid; i < len; i += THREADS) newest = max(newest, r.time[i]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) newest = max(newest, __shfl_xor(newest, d));
    if (lane == 0) s_part[wave] = newest;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) newest = max(newest, s_part[w]);
    r.newest = (long)newest - a.j.window;
    int recent = 0;
    for (int i = tid; i < len; i += THREADS) recent += r.recent(i);
    recent = block_sum(recent, s_part);
    r.by_time = recent >= budget;

    // the rank of the last token that is kept (`least`), and how many of that rank are
    int left = r.by_time ? budget : budget - recent;
    uint32_t least = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = tid; i < 256 * COPIES; i += THREADS) hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < len; i += THREADS) {
            bool in;
            const uint32_t k = r.rank(i, &in);
            if (in && (shift == 24 || (k ^ least) >> (shift + 8) == 0))
                atomicAdd(&hist[((k >> shift) & 255) * COPIES + (lane & (COPIES - 1))], 1);
        }
        __syncthreads();
        if (tid < 256) {
            int sum = 0;
            for (int x = 0; x < COPIES; ++x) sum += hist[tid * COPIES + ((x + tid) & (COPIES - 1))];
            s_bin[tid] = sum;
        }
        __syncthreads();
        if (wave == 0) {
            // from the highest byte down: lane takes four
            int n[4], sum = 0;
#pragma unroll
            for (int x = 0; x < 4; ++x) sum += n[x] = s_bin[255 - 4 * lane - x];
            int above = sum;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int up = __shfl_up(above, d);
                if (lane >= d) above += up;
            }
            above -= sum;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if (above < left && above + n[x] >= left) { s_pick = 255 - 4 * lane - x; s_left = left - above; }
                above += n[x];
            }
        }
        __syncthreads();
        least |= (uint32_t)s_pick << shift;
        left = s_left;
    }

    // a wavefront's stretch of slots
    const int per = (len + THREADS - 1) / THREADS * 64, from = wave * per < len ? wave * per : len, to = from + per < len ? from + per : len;
    auto state = [&](int i, bool* equal) {                  // kept whatever the others of the last rank do
        bool in;
        const uint32_t k = r.rank(i, &in);
        *equal = in && k == least;
        return !in || k > least;
    };
    int equals = 0;
    for (int i0 = from; i0 < to; i0 += 64) {
        bool equal = false;
        if (i0 + lane < to) state(i0 + lane, &equal);
        equals += __popcll(__ballot(equal));
    }
    __syncthreads();
    if (lane == 0) s_part[wave] = equals;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += s_part[w];
    const unsigned long long below = (1ull << lane) - 1;
    int holes = 0, movers = 0;
    for (int pass = 0; pass < 2; ++pass) {
        int run = before;
        if (pass == 1) {
            if (lane == 0) { s_hole[wave] = holes; s_mover[wave] = movers; }
            __syncthreads();
            holes = movers = 0;
            for (int w = 0; w < wave; ++w) { holes += s_hole[w]; movers += s_mover[w]; }
        }
        for (int i0 = from; i0 < to; i0 += 64) {
            const int i = i0 + lane;
            bool equal = false, kept = false;
            if (i < to) kept = state(i, &equal);
            const unsigned long long eq = __ballot(equal);
            if (equal) kept = run + __popcll(eq & below) < left;
            run += __popcll(eq);
            const bool hole = i < to && !kept && i < budget, mover = kept && i >= budget;
            const unsigned long long hb = __ballot(hole), mb = __ballot(mover);
            if (pass == 1) {
                if (hole) a.hole[at + holes + __popcll(hb & below)] = i;
                if (mover) a.mover[at + movers + __popcll(mb & below)] = i;
                if (a.copies && kept && i < budget) {
                    c.weight[at + i] = r.weight[i];
                    c.time[at + i] = r.time[i];
                }
            }
            holes += __popcll(hb);
            movers += __popcll(mb);
        }
    }
    if (wave == WAVES - 1 && lane == 0) a.count[pair] = movers;
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
    uint4 *k = (uint4*)c.k, *v = (uint4*)c.v;
    for (long i = blockIdx.x * 256 + threadIdx.x; i < (long)n * pieces; i += gridDim.x * 256) {
        const int m = (int)(i / pieces), p = (int)(i - (long)m * pieces);
        const int from = a.mover[at + m], to = a.hole[at + m];
        const long src = row(from), dst = row(to);
        if (src >= 0 && dst >= 0) {
            const uint4 x = k[src + p], y = v[src + p];
            k[dst + p] = x;
            v[dst + p] = y;
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
    hipLaunchKernelGGL(select_kernel, dim3(c.heads, c.seqs), dim3(THREADS), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // workgroups of the moves: a few for each compute unit, no more than the most there can be to move
    const long most = ((long)(c.capacity - j.budget < j.budget ? c.capacity - j.budget : j.budget) * (c.dim * (c.bf16 ? 2 : 4) / 16) + 255) / 256;
    long per = (8L * device_units() + pairs - 1) / pairs;
    per = per > most ? most : per;
    hipLaunchKernelGGL(move_kernel, dim3((unsigned)(per < 1 ? 1 : per), c.heads, c.seqs), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace cb
