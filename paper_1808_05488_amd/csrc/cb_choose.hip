// Which pages of a cache a query has to read: bounds of every page's keys, scores from them, the highest ones.
//
// Bounds.  For a page and key head the smallest and the largest of its tokens' keys, value by value.  Only pages with new tokens are gone through;
// memory bounds it (their keys).  A cache in 8 bits has bounds in bfloat16, rounded outwards where its scales are no powers of two.
//
// Scores.  sum_d max(q_d lo_d, q_d hi_d) is no less than q.k for any key k of the page; a page's score is the largest of its key head's query heads.  Sums
// are in float64 and rounded to float32 once, so that what is chosen does not depend on their order (products of float32 values are exact there); four lanes a page,
// each of which reads every fourth 16 bytes of its bounds.  Memory bounds it: 2 * dim values a page and key head.
//
// Choice.  A workgroup for every (sequence, key head) finds the lowest score that is taken by counting digits (radix selection, ten bits a pass
// between the lowest and the highest score), then lists the pages in order.  Sequences whose pages are all taken need no scores.
#include "cb_tokens.h"

namespace cb {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct ChooseArgs {
    ChooseJob j;
    Cache c;
    int group;
    float* scores;                       // of (sequence, key head): pitch max_pages
};

__device__ __forceinline__ int pages_of(const Cache& c, int seq)
{
    return (clamp_length(c.lengths[seq], c.capacity) + (1 << c.page_shift) - 1) >> c.page_shift;
}

// The units of all sequences in order, n(sequence) each: the sequence that unit u belongs to and its number there; -1: there are fewer.  For all lanes of a wavefront.
struct Found { int seq; long unit; };
template <typename N> __device__ __forceinline__ Found find_unit(const Cache& c, long u, N n)
{
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < c.seqs; s0 += 64) {
        // (units of 64 sequences may pass 32 bits: they are added up in 64)
        long sum = s0 + lane < c.seqs ? n(s0 + lane) : 0;
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
            const long before = __shfl_up(sum, i);
            if (lane >= i) sum += before;
        }
        const unsigned long long past = __ballot(sum > u);
        if (past) {
            const int at = __builtin_ctzll(past);
            const long before = at > 0 ? __shfl(sum, at - 1) : 0;
            return Found{s0 + at, u - before};
        }
        u -= __shfl(sum, 63);
    }
    return Found{-1, 0};
}

// ---------------------------------------------------------------- bounds
constexpr int BOUND_THREADS = 256;

template <typename KT> struct Piece { static constexpr int N = 16 / sizeof(KT); };       // values of 16 bytes
__device__ __forceinline__ void widen_piece(const u32x4& w, float (&f)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ void widen_piece(const u32x4& w, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ void widen_piece(const u32x4& w, float (&f)[16])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[4 * i] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 0);
        f[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 1);
        f[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 2);
        f[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 3);
    }
}
// To bfloat16, up or down; what is not a number stays so.
__device__ __forceinline__ uint16_t outwards(float f, bool up)
{
    const uint32_t b = __float_as_uint(f);
    if (f != f) return 0x7FC0;
    const bool away = (b & 0xFFFFu) != 0 && up == ((b >> 31) == 0);      // from zero
    return (uint16_t)((b >> 16) + (away ? 1 : 0));
}

template <typename KT>
__global__ __launch_bounds__(BOUND_THREADS) void bound_kernel(const int32_t* since, const Cache c)
{
    constexpr int N = Piece<KT>::N;
    __shared__ float s_lo[BOUND_THREADS * N], s_hi[BOUND_THREADS * N];
    const int tid = threadIdx.x, per_row = c.dim / N, teams = BOUND_THREADS / per_row, team = tid / per_row, sub = tid - team * per_row;
    auto first_page = [&](int s) {
        const int pages = pages_of(c, s), from = since ? clamp_length(since[s], c.capacity) >> c.page_shift : 0;
        return from < pages ? from : pages;
    };
    for (long u = blockIdx.x;; u += gridDim.x) {
        const Found f = find_unit(c, u, [&](int s) { return (long)(pages_of(c, s) - first_page(s)) * c.heads; });
        if (f.seq < 0) return;
        const int at = (int)(f.unit / c.heads), h = (int)(f.unit - (long)at * c.heads), p = first_page(f.seq) + at;
        const int page = c.table[(long)f.seq * c.max_pages + p], left = clamp_length(c.lengths[f.seq], c.capacity) - (p << c.page_shift);
        if ((unsigned)page >= (unsigned)c.n_pages) continue;
        const int rows = left < 1 << c.page_shift ? left : 1 << c.page_shift;
        const long head = (long)page * c.heads + h;
        const KT* src = (const KT*)c.k + (head << c.page_shift) * c.dim + sub * N;
        const float* scale = c.k_scale + (head << (c.page_shift - 4));
        float lo[N], hi[N];
#pragma unroll
        for (int i = 0; i < N; ++i) { lo[i] = __builtin_inff(); hi[i] = -__builtin_inff(); }
        if (team < teams) {
#pragma unroll 4
            for (int r = team; r < rows; r += teams) {
                float x[N];
                widen_piece(*reinterpret_cast<const u32x4*>(src + (long)r * c.dim), x);
                if constexpr (sizeof(KT) == 1) {
                    const float y = scale[r >> 4];
#pragma unroll
                    for (int i = 0; i < N; ++i) x[i] *= y;
                }
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    lo[i] = x[i] < lo[i] || x[i] != x[i] ? x[i] : lo[i];
                    hi[i] = x[i] > hi[i] || x[i] != x[i] ? x[i] : hi[i];
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                s_lo[team * c.dim + sub * N + i] = lo[i];
                s_hi[team * c.dim + sub * N + i] = hi[i];
            }
        }
        __syncthreads();
        const int used = teams < rows ? teams : rows;
        for (int d = tid; d < 2 * c.dim; d += BOUND_THREADS) {
            const bool up = d >= c.dim;
            const float* s = up ? s_hi + d - c.dim : s_lo + d;
            float y = s[0];
            for (int t = 1; t < used; ++t) {
                const float x = s[t * c.dim];
                y = (up ? x > y : x < y) || x != x ? x : y;
            }
            const long to = head * 2 * c.dim + d;
            if constexpr (sizeof(KT) == 1) ((uint16_t*)c.bounds)[to] = outwards(y, up);
            else if constexpr (sizeof(KT) == 2) narrow(y, ((uint16_t*)c.bounds)[to]);
            else ((float*)c.bounds)[to] = y;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- scores
constexpr int SCORE_THREADS = 256, SCORE_PAGES = SCORE_THREADS / 4, SCORE_HEADS = 4;       // query heads at a time

template <typename BT, typename T>
__global__ __launch_bounds__(SCORE_THREADS) void score_kernel(const ChooseArgs a)
{
    constexpr int N = Piece<BT>::N;
    __shared__ __align__(16) float s_q[SCORE_HEADS][256];
    const Cache& c = a.c;
    const int tid = threadIdx.x, quarter = tid & 3, pieces = c.dim / N;
    auto chunks = [&](int s) {
        const int pages = pages_of(c, s);
        return pages <= a.j.budget ? 0 : (pages + SCORE_PAGES - 1) / SCORE_PAGES;
    };
    for (long u = blockIdx.x;; u += gridDim.x) {
        const Found f = find_unit(c, u, [&](int s) { return (long)chunks(s) * c.heads; });
        if (f.seq < 0) return;
        const int n = chunks(f.seq), h = (int)(f.unit / n), p = (int)(f.unit - (long)h * n) * SCORE_PAGES + (tid >> 2), pages = pages_of(c, f.seq);
        int page = -1;
        if (p < pages) page = c.table[(long)f.seq * c.max_pages + p];
        const bool there = (unsigned)page < (unsigned)c.n_pages;
        const BT* bounds = (const BT*)c.bounds + (there ? ((long)page * c.heads + h) * 2 * c.dim : 0);
        float best = -__builtin_inff();
        for (int g0 = 0; g0 < a.group; g0 += SCORE_HEADS) {
            __syncthreads();
            for (int i = tid; i < SCORE_HEADS * c.dim; i += SCORE_THREADS) {
                const int g = i / c.dim, d = i - g * c.dim, head = h * a.group + (g0 + g < a.group ? g0 + g : g0);
                s_q[g][d] = widen(((const T*)a.j.q.data)[(long)f.seq * a.j.q.token + (long)head * a.j.q.head + d]);
            }
            __syncthreads();
            double sum[SCORE_HEADS] = {};
            if (there)
                for (int i = quarter; i < pieces; i += 4) {
                    float lo[N], hi[N];
                    widen_piece(*reinterpret_cast<const u32x4*>(bounds + i * N), lo);
                    widen_piece(*reinterpret_cast<const u32x4*>(bounds + c.dim + i * N), hi);
#pragma unroll
                    for (int g = 0; g < SCORE_HEADS; ++g)
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            const float q = s_q[g][i * N + e];
                            sum[g] = __builtin_fma((double)q, (double)(q >= 0.0f ? hi[e] : lo[e]), sum[g]);
                        }
                }
#pragma unroll
            for (int g = 0; g < SCORE_HEADS; ++g) {
                sum[g] += __shfl_xor(sum[g], 1);
                sum[g] += __shfl_xor(sum[g], 2);
                const float score = (float)sum[g];
                best = score != score ? __builtin_inff() : fmaxf(best, score);       // (what is not a number rules nothing out)
            }
        }
        // (a page without a number holds no token: it comes last)
        if (p < pages && quarter == 0) a.scores[((long)f.seq * c.heads + h) * c.max_pages + p] = there ? best : -__builtin_inff();
    }
}

// ---------------------------------------------------------------- choice
constexpr int THREADS = 1024, WAVES = THREADS / 64, DIGIT = 10, BINS = 1 << DIGIT;
constexpr int LDS_RANKS = 16384;
static_assert(BINS == THREADS, "a bin a thread");

// Sum over the threads before this one, and over all.
__device__ __forceinline__ int sum_before(int v, int* s_part, int* all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sum = wave_scan(v);
    if (lane == 63) s_part[wave] = sum;
    __syncthreads();
    const int parts = wave_scan(lane < WAVES ? s_part[lane] : 0);
    *all = __builtin_amdgcn_readlane(parts, 63);
    const int before = __shfl(parts, wave > 0 ? wave - 1 : 0);
    __syncthreads();
    return sum - v + (wave > 0 ? before : 0);
}

__global__ __launch_bounds__(THREADS) void choose_kernel(const ChooseArgs a, int room)
{
    extern __shared__ uint32_t s_rank[];
    __shared__ int hist[BINS], s_part[WAVES], s_pick[3];
    __shared__ uint32_t s_low, s_high;
    const Cache& c = a.c;
    const int seq = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 63, budget = a.j.budget;
    const long pair = (long)seq * c.heads + h;
    const int n = pages_of(c, seq);
    int32_t* chosen = a.j.chosen + pair * budget;
    if (n <= budget) {
        for (int i = tid; i < budget; i += THREADS) chosen[i] = i < n ? i : -1;
        if (tid == 0) a.j.count[pair] = n;
        return;
    }
    const float* scores = a.scores + pair * c.max_pages;
    const bool in_lds = n <= room;
    // ranks in the scores' order, above all of them the pages that are always taken
    auto made = [&](int i) {
        if (i < a.j.first || i >= n - a.j.recent) return 0xFFFFFFFFu;
        const uint32_t b = __float_as_uint(scores[i] + 0.0f);
        return b & 0x80000000u ? ~b : b | 0x80000000u;
    };
    auto rank = [&](int i) { return in_lds ? s_rank[i] : made(i); };
    if (tid == 0) { s_low = 0xFFFFFFFFu; s_high = 0; }
    __syncthreads();
    uint32_t low = 0xFFFFFFFFu, high = 0;
#pragma unroll 4
    for (int i = tid; i < n; i += THREADS) {
        const uint32_t r = made(i);
        if (in_lds) s_rank[i] = r;
        low = min(low, r);
        high = max(high, r == 0xFFFFFFFFu ? 0u : r);
    }
    low = ~wave_max_unsigned(~low);
    high = wave_max_unsigned(high);
    if (lane == 0) { atomicMin(&s_low, low); atomicMax(&s_high, high); }
    __syncthreads();
    low = s_low;
    high = s_high;
    // `want` of those that rank low .. high are taken, all that rank above are.  (Those that are always taken are fewer than the budget, or
    // as many: then none of the others is.)
    const int forced = a.j.first + a.j.recent;
    int want = budget - forced;
    bool found = want == 0;
    if (found) low = high = 0xFFFFFFFEu;
    while (!found) {
        const int bits = 32 - __builtin_clz((high - low) | 1u), shift = bits > DIGIT ? bits - DIGIT : 0;
        hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += THREADS) {
            const uint32_t r = rank(i);
            if (r >= low && r <= high) atomicAdd(&hist[(r - low) >> shift], 1);
        }
        __syncthreads();
        const int bin = BINS - 1 - tid, here = hist[bin];
        int all;
        const int above = sum_before(here, s_part, &all);
        if (above < want && above + here >= want) { s_pick[0] = bin; s_pick[1] = above; s_pick[2] = here; }
        __syncthreads();
        low += (uint32_t)s_pick[0] << shift;
        const uint32_t end = low + ((1u << shift) - 1u);
        high = end < high ? end : high;
        want -= s_pick[1];
        found = shift == 0 || want == s_pick[2];
        __syncthreads();
    }
    // the pages in order, a stretch of them a thread
    const int each = (n + THREADS - 1) / THREADS, begin = tid * each < n ? tid * each : n, end = begin + each < n ? begin + each : n;
    int sure = 0, equal = 0, all;
    for (int i = begin; i < end; ++i) {
        const uint32_t r = rank(i);
        sure += r > high;
        equal += r >= low && r <= high;
    }
    int before = sum_before(sure, s_part, &all), ties = sum_before(equal, s_part, &all);
    for (int i = begin; i < end; ++i) {
        const uint32_t r = rank(i);
        if (r > high) chosen[before++ + (ties < want ? ties : want)] = i;
        else if (r >= low) {
            if (ties < want) chosen[before + ties] = i;
            ++ties;
        }
    }
    if (tid == 0) a.j.count[pair] = budget;
}

unsigned grid_for(long most, long per_unit)
{
    const long want = per_unit * device_units();
    return (unsigned)(most < want ? (most < 1 ? 1 : most) : want);
}

}  // namespace

hipError_t launch_bound(const int32_t* since, const Cache& c, hipStream_t st)
{
    const dim3 grid(grid_for((long)c.seqs * c.heads * c.max_pages, 8)), block(BOUND_THREADS);
    if (c.e4m3) hipLaunchKernelGGL(bound_kernel<uint8_t>, grid, block, 0, st, since, c);
    else if (c.bf16) hipLaunchKernelGGL(bound_kernel<uint16_t>, grid, block, 0, st, since, c);
    else hipLaunchKernelGGL(bound_kernel<float>, grid, block, 0, st, since, c);
    return hipGetLastError();
}

hipError_t launch_choose(const ChooseJob& j, const Cache& c, hipStream_t st)
{
    ChooseArgs a;
    a.j = j;
    a.c = c;
    a.group = j.q.heads / c.heads;
    a.scores = reinterpret_cast<float*>(c.scratch + scratch_plan(c, 0).pages);
    if (j.budget < c.max_pages) {
        const dim3 grid(grid_for((long)c.seqs * c.heads * ((c.max_pages + SCORE_PAGES - 1) / SCORE_PAGES), 8)), block(SCORE_THREADS);
        if (c.e4m3) {
            if (c.bf16) hipLaunchKernelGGL((score_kernel<uint16_t, uint16_t>), grid, block, 0, st, a);
            else hipLaunchKernelGGL((score_kernel<uint16_t, float>), grid, block, 0, st, a);
        } else if (c.bf16) hipLaunchKernelGGL((score_kernel<uint16_t, uint16_t>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((score_kernel<float, float>), grid, block, 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int room = c.max_pages < LDS_RANKS ? c.max_pages : LDS_RANKS;
    hipLaunchKernelGGL(choose_kernel, dim3(c.heads, c.seqs), dim3(THREADS), (size_t)room * 4, st, a, room);
    return hipGetLastError();
}

}  // namespace cb
