// Attention of one new token per sequence over a paged key-value cache.
//
// For each sequence and key head: s_j = scale q.k_j for the query heads that read the key head, the softmax over the
// cached tokens j, and the weighted sum of the v_j.  Keys and values are read once, so memory bounds it: 4 * dim * heads operations for
// 2 * dim * heads / group values.  One pass: every wavefront takes tiles of consecutive tokens and keeps, for up to 16 query heads, the running maximum m,
// the sum l of e^(s - m) and the sum o of e^(s - m) v; a tile with a larger maximum scales l and o by e^(m - m').  Parts of a sequence (wavefronts of
// a workgroup, then workgroups) are joined the same way.
//
// Layout.  S^T = K Q^T and O^T = V^T P^T on the matrix cores, 16 query heads as columns.  A lane's column is its query head (lane & 15) in both, so
// that m and l live in the lane that needs them, and what S^T leaves in a lane -- the scores of tokens 4 * (lane >> 4) + r -- is
// what P^T wants there, if the tokens of a tile are numbered to suit; no value changes lanes but for the maximum.  Keys and values come
// from memory into registers as the matrix cores take them, whole rows by neighbouring lanes.
//
// Work is split over the length.  A unit is UNIT tokens of a (sequence, key head, block of query heads); the units of all of them,
// in order, are dealt to the workgroups in equal runs, whatever the lengths, which the kernel reads itself.  A run's end in the middle of a
// (sequence, head) leaves a part in the scratch buffer, and the workgroup that comes last joins the parts, in order.
#include "cb_tokens.h"

namespace cb {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr float LOWEST = -3.402823466e38f;       // of a maximum, so that nothing is subtracted from minus infinity
constexpr int ROWS = ATTEND_ROWS;
constexpr int UNIT = 256;

struct AttendArgs {
    AttendJob j;
    Cache c;
    int group, blocks;             // query heads of a key head, blocks of ROWS of them
    int q_aligned;
    int* counters;
    float *parts, *lse, *scores;
    int pitch;                     // of a query head's scores
};

// e^x for the difference x of two scores, which is exact or nearly so; scores times log2 e would be rounded at their own size.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

// Part of (sequence, key head, block of query heads) in the scratch buffer: ROWS maxima, ROWS sums, ROWS x DP values.
template <int DP> constexpr int part_floats() { return ROWS * (DP + 2); }

__device__ __forceinline__ void put(float* at, float a, float b)
{
    const unsigned long long w = (unsigned long long)__float_as_uint(b) << 32 | __float_as_uint(a);
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(at), w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get(const float* at)
{
    const unsigned long long w = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((unsigned)w), __uint_as_float((unsigned)(w >> 32)));
}

// The units of the sequences in order, and who has them.  All of it is the same for every lane of a wavefront.
struct Units {
    const int32_t* lengths;
    int seqs, capacity, per_seq;       // per_seq: (key head, block) pairs of a sequence
    __device__ int of(int len) const { return len > UNIT ? (len + UNIT - 1) / UNIT : 1; }
    __device__ int at(int s) const { return of(clamp_length(lengths[s], capacity)) * per_seq; }
    __device__ int total() const
    {
        const int lane = threadIdx.x & 63;
        int sum = 0;
        for (int s = lane; s < seqs; s += 64) sum += at(s);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        return __builtin_amdgcn_readfirstlane(sum);
    }
    // the sequence that unit u belongs to, and its first unit
    __device__ int find(int u, int* first) const
    {
        const int lane = threadIdx.x & 63;
        int before = 0;
        for (int s0 = 0; s0 < seqs; s0 += 64) {
            int sum = s0 + lane < seqs ? at(s0 + lane) : 0;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int up = __shfl_up(sum, d);
                if (lane >= d) sum += up;
            }
            const unsigned long long past = __ballot(before + sum > u);
            if (past) {
                const int at = __builtin_ctzll(past);
                *first = before + (at > 0 ? __builtin_amdgcn_readlane(sum, at - 1) : 0);
                return s0 + at;
            }
            before += __builtin_amdgcn_readlane(sum, 63);
        }
        *first = before;
        return seqs;
    }
};

// n units dealt to w workgroups: the first n % w get one more than the others.
struct Deal {
    unsigned each, more;
    __device__ Deal(unsigned n, unsigned w) : each(n / w), more(n % w) {}
    __device__ unsigned first(unsigned g) const { return g * each + (g < more ? g : more); }
    __device__ unsigned owner(unsigned u) const
    {
        const unsigned big = more * (each + 1);
        return u < big ? u / (each + 1) : more + (u - big) / each;
    }
};

// How a type's tiles look.  PE: consecutive values of a row that a lane takes of V, NP such pieces 16 * PE apart.
template <typename T, int DP> struct Tile;
template <int DP> struct Tile<uint16_t, DP> {
    static constexpr int WAVES = DP == 256 ? 4 : 8;      // of a workgroup: as many as its registers have room for
    static constexpr int TOKENS = 32, PE = DP == 64 ? 4 : 8, NP = DP / (16 * PE);
    static constexpr int KSTEPS = DP / 32;       // of S^T: 32 values of a head a step
};
template <int DP> struct Tile<float, DP> {
    static constexpr int WAVES = DP == 256 ? 4 : 8;
    static constexpr int TOKENS = 16, PE = 4, NP = DP / (16 * PE);
    static constexpr int KSTEPS = DP / 16;       // four steps of 4 values
};

// A wavefront's pages: lane x has that of its sub-tile x (16 tokens) of the next 64.
template <int SUB, int WAVES> __device__ __forceinline__ int load_pages(const int32_t* table, int shift, int n_pages, int tile, int len)
{
    const int lane = threadIdx.x & 63, tok = (tile + lane / SUB * WAVES) * SUB * 16 + lane % SUB * 16;
    int page = -1;
    if (tok < len) page = table[tok >> shift];
    return (unsigned)page < (unsigned)n_pages ? page : -1;
}

template <typename V> __device__ __forceinline__ V load_once(const void* p) { return __builtin_nontemporal_load(reinterpret_cast<const V*>(p)); }

template <typename T, int DP>
__global__ __launch_bounds__((Tile<T, DP>::WAVES * 64)) void attend_kernel(const AttendArgs a)
{
    constexpr bool HALF = sizeof(T) == 2;
    typedef Tile<T, DP> TL;
    constexpr int WAVES = TL::WAVES, THREADS = WAVES * 64, SUB = TL::TOKENS / 16, NP = TL::NP, PE = TL::PE, KSTEPS = TL::KSTEPS;
    constexpr int ROUNDS = UNIT / (WAVES * TL::TOKENS);                // tiles of a wavefront in a unit
    constexpr int DW = PE * (int)sizeof(T) / 4;                        // 32-bit words of a piece
    typedef uint32_t piece_t __attribute__((ext_vector_type(DW)));
    typedef uint32_t key_t __attribute__((ext_vector_type(4)));
    __shared__ float s_o[WAVES][ROWS][DP + 4];
    __shared__ float s_m[WAVES][ROWS], s_l[WAVES][ROWS];
    __shared__ int s_last;

    const Cache& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, quad = lane >> 4;
    const int D = c.dim, per_seq = c.heads * a.blocks;
    const Units units{c.lengths, c.seqs, c.capacity, per_seq};
    const unsigned total = units.total(), groups = total < gridDim.x ? total : gridDim.x;
    if (blockIdx.x >= groups) return;
    const Deal deal(total, groups);
    int u = deal.first(blockIdx.x);
    const int end = deal.first(blockIdx.x + 1);

    int first;
    int seq = units.find(u, &first);
    while (u < end && seq < c.seqs) {
        const int len = clamp_length(c.lengths[seq], c.capacity), nu = units.of(len);
        const int pair = (unsigned)(u - first) / (unsigned)nu, from = u - first - pair * nu;
        const int to = nu - from < end - u ? nu : from + (end - u);
        const int h = (unsigned)pair / (unsigned)a.blocks, blk = pair - h * a.blocks;
        const int row0 = blk * ROWS, rows = a.group - row0 < ROWS ? a.group - row0 : ROWS;
        const int32_t* table = c.table + (long)seq * c.max_pages;

        // this wavefront's tiles: t, t + WAVES, ... below t1
        int t = from * (ROUNDS * WAVES) + wave;
        const int t1 = to * (ROUNDS * WAVES) < (len + TL::TOKENS - 1) / TL::TOKENS ? to * (ROUNDS * WAVES) : (len + TL::TOKENS - 1) / TL::TOKENS;
        int pages = load_pages<SUB, WAVES>(table, c.page_shift, c.n_pages, t, len), ahead = -1, used = 0;
        if (t + 64 / SUB * WAVES < t1) ahead = load_pages<SUB, WAVES>(table, c.page_shift, c.n_pages, t + 64 / SUB * WAVES, len);

        // this lane's part of the query heads: head l16, values 32 * i + 8 * quad .. (or 16 * i + 4 * quad ..)
        key_t q[KSTEPS];
        {
            const T* src = (const T*)a.j.q.data + (long)seq * a.j.q.token + (long)(h * a.group + row0 + l16) * a.j.q.head;
            constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
            for (int i = 0; i < KSTEPS; ++i) {
                const int d = (4 * i + quad) * E;
                q[i] = key_t(0);
                if (l16 < rows && d < D) {
                    if (a.q_aligned) q[i] = *reinterpret_cast<const key_t*>(src + d);
                    else {
                        T e[E];
#pragma unroll
                        for (int x = 0; x < E; ++x) e[x] = src[d + x];
                        __builtin_memcpy(&q[i], e, 16);
                    }
                }
            }
        }
        float m = LOWEST, l = 0.0f;
        f32x4 o[NP * PE];
#pragma unroll
        for (int i = 0; i < NP * PE; ++i) o[i] = f32x4{0, 0, 0, 0};

        key_t k[SUB][KSTEPS];
        piece_t v[SUB][4][NP];
        // tile x: where its sub-tiles' rows are (in values), how many tokens they hold
        struct Where { long at[SUB]; int left[SUB]; };
        auto find = [&](int x, int slot) {
            Where w;
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                const int tok = x * TL::TOKENS + 16 * s, page = __builtin_amdgcn_readlane(pages, slot * SUB + s);
                w.left[s] = page >= 0 ? (len - tok < 16 ? len - tok : 16) : 0;
                w.at[s] = page >= 0 ? ((((long)page * c.heads + h) << c.page_shift) + (tok & ((1 << c.page_shift) - 1))) * D : 0;
            }
            return w;
        };
        auto load_k = [&](const Where& w) {
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                const T* src = (const T*)c.k + w.at[s] + l16 * D;
#pragma unroll
                for (int i = 0; i < KSTEPS; ++i) {
                    const int d = (4 * i + quad) * (16 / (int)sizeof(T));
                    k[s][i] = key_t(0);
                    if (l16 < w.left[s] && d < D) k[s][i] = load_once<key_t>(src + d);
                }
            }
        };
        auto load_v = [&](const Where& w) {
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                const T* src = (const T*)c.v + w.at[s] + 4 * quad * D;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        const int d = (16 * p + l16) * PE;
                        v[s][r][p] = piece_t(0);
                        if (4 * quad + r < w.left[s] && d < D) v[s][r][p] = load_once<piece_t>(src + r * D + d);
                    }
            }
        };
        Where here, next;
        if (t < t1) {
            here = find(t, 0);
            load_k(here);
            load_v(here);
        }
        for (; t < t1; t += WAVES) {
            // scores of tokens 16 * s + 4 * quad + r for query head l16
            f32x4 sc[SUB];
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                sc[s] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < KSTEPS; ++i) {
                    if constexpr (HALF)
                        sc[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[s][i]), __builtin_bit_cast(bf16x8, q[i]), sc[s], 0, 0, 0);
                    else {
                        const f32x4 x = __builtin_bit_cast(f32x4, k[s][i]), y = __builtin_bit_cast(f32x4, q[i]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[s] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], sc[s], 0, 0, 0);
                    }
                }
            }
            // the next tile's keys come while this one's weights are made, its values while the next one's scores are
            const bool more = t + WAVES < t1;
            if (more) {
                if (++used == 64 / SUB) {
                    used = 0;
                    pages = ahead;
                    if (t + (1 + 64 / SUB) * WAVES < t1) ahead = load_pages<SUB, WAVES>(table, c.page_shift, c.n_pages, t + (1 + 64 / SUB) * WAVES, len);
                }
                next = find(t + WAVES, used);
                load_k(next);
            }
            float top = LOWEST;
#pragma unroll
            for (int s = 0; s < SUB; ++s)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float x = sc[s][r] * a.j.scale;
                    if (a.j.softcap > 0.0f) x = a.j.softcap * tanhf(x / a.j.softcap);
                    x = 4 * quad + r < here.left[s] ? x : -__builtin_inff();
                    sc[s][r] = x;
                    top = fmaxf(top, x);
                }
            if (a.scores && l16 < rows) {
                float* to_scores = a.scores + ((long)seq * a.j.q.heads + h * a.group + row0 + l16) * a.pitch + t * TL::TOKENS + 4 * quad;
#pragma unroll
                for (int s = 0; s < SUB; ++s)
                    if (t * TL::TOKENS + 16 * s < a.pitch) *reinterpret_cast<f32x4*>(to_scores + 16 * s) = sc[s];
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (top > m) {
                const float scale = exp_of(m - top);
                m = top;
                l *= scale;
#pragma unroll
                for (int i = 0; i < NP * PE; ++i) o[i] *= scale;
            }
            float p[SUB][4];
#pragma unroll
            for (int s = 0; s < SUB; ++s)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    p[s][r] = exp_of(sc[s][r] - m);
                    l += p[s][r];
                }
            if constexpr (HALF) {
                // P in two bfloat16 terms: one alone would round as much as the result's own rounding does
                bf16x8 hi, lo;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    hi[x] = (__bf16)p[x / 4][x % 4];
                    lo[x] = (__bf16)(p[x / 4][x % 4] - (float)hi[x]);
                }
#pragma unroll
                for (int pc = 0; pc < NP; ++pc)
#pragma unroll
                    for (int e = 0; e < PE; ++e) {
                        // value e of the eight tokens, in the order that P has them in
                        uint32_t w[4];
                        const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int s = x / 2, r = 2 * (x % 2);
                            w[x] = __builtin_amdgcn_perm(v[s][r + 1][pc][e / 2], v[s][r][pc][e / 2], sel);
                        }
                        const bf16x8 vt = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
                        o[pc * PE + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, hi, o[pc * PE + e], 0, 0, 0);
                        o[pc * PE + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, lo, o[pc * PE + e], 0, 0, 0);
                    }
            } else {
#pragma unroll
                for (int pc = 0; pc < NP; ++pc)
#pragma unroll
                    for (int e = 0; e < PE; ++e)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            o[pc * PE + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[0][r][pc][e]), p[0][r], o[pc * PE + e], 0, 0, 0);
            }
            if (more) {
                load_v(next);
                here = next;
            }
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);

        // join the wavefronts: lane has o of query head l16, values (16 * p + 4 * quad + r) * PE + e
        __syncthreads();
        if (quad == 0) { s_m[wave][l16] = m; s_l[wave][l16] = l; }
        if (l16 < rows) {
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int e = 0; e < PE; ++e) s_o[wave][l16][(16 * p + 4 * quad + r) * PE + e] = o[p * PE + e][r];
        }
        __syncthreads();

        const long q_head = (long)seq * a.j.q.heads + h * a.group + row0;
        // row, values d and d + 1: x and y over L
        auto finish = [&](int row, int d, float M, float L, float x, float y) {
            const float inv = L == 0.0f ? 0.0f : 1.0f / L;
            if (d < D) {
                T* out = (T*)a.j.out.data + (long)seq * a.j.out.token + (long)(h * a.group + row0 + row) * a.j.out.head + d;
                T e0, e1;
                narrow(x * inv, e0);
                narrow(y * inv, e1);
                out[0] = e0;
                out[1] = e1;
            }
            if (d == 0) {
                const float z = L == 0.0f ? -__builtin_inff() : M + __builtin_amdgcn_logf(L) * LN2;
                if (a.j.lse) a.j.lse[q_head + row] = z;
                a.lse[q_head + row] = z;
            }
        };
        // what the wavefronts have of row, values d and d + 1
        auto join = [&](int row, int d, float* M, float* L, float* x, float* y) {
            *M = LOWEST;
            *L = *x = *y = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) *M = fmaxf(*M, s_m[w][row]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = exp_of(s_m[w][row] - *M);
                *L += f * s_l[w][row];
                *x += f * s_o[w][row][d];
                *y += f * s_o[w][row][d + 1];
            }
        };
        const bool whole = from == 0 && to == nu;
        float* mine = a.parts + (2L * blockIdx.x + (from == 0 ? 1 : 0)) * part_floats<DP>();
        for (int i = 2 * tid; i < rows * DP; i += 2 * THREADS) {
            const int row = i / DP, d = i % DP;
            float M, L, x, y;
            join(row, d, &M, &L, &x, &y);
            if (whole) finish(row, d, M, L, x, y);
            else {
                put(mine + 2 * ROWS + i, x, y);
                if (d == 0) put(mine + 2 * row, M, L);
            }
        }
        if (!whole) {
            __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0): this wavefront's stores are where every compute unit sees them
            __syncthreads();
            // the workgroups that share this pair; the first of them has no other pair that goes on behind it
            const unsigned u0 = first + pair * nu, w0 = deal.owner(u0), w1 = deal.owner(u0 + nu - 1);
            if (tid == 0) {
                s_last = __hip_atomic_fetch_add(a.counters + w0, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)(w1 - w0);
                if (s_last) __hip_atomic_store(a.counters + w0, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (s_last) {
                // each wavefront takes every WAVES-th part, in order; then the wavefronts are joined as before
                for (int i = 2 * lane; i < rows * DP; i += 128) {
                    const int row = i / DP, d = i % DP;
                    float M = LOWEST, L = 0.0f, x = 0.0f, y = 0.0f;
                    for (unsigned w = w0 + wave; w <= w1; w += 4 * WAVES) {
                        float2 ml[4], xy[4];
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            const unsigned g = w + n * WAVES;
                            const float* part = a.parts + (2L * g + (g == w0 ? 1 : 0)) * part_floats<DP>();
                            ml[n] = make_float2(LOWEST, 0.0f);
                            xy[n] = make_float2(0.0f, 0.0f);
                            if (g <= w1) { ml[n] = get(part + 2 * row); xy[n] = get(part + 2 * ROWS + i); }
                        }
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            const float top = fmaxf(M, ml[n].x), f = exp_of(M - top), g = exp_of(ml[n].x - top);
                            M = top;
                            L = f * L + g * ml[n].y;
                            x = f * x + g * xy[n].x;
                            y = f * y + g * xy[n].y;
                        }
                    }
                    s_o[wave][row][d] = x;
                    s_o[wave][row][d + 1] = y;
                    if (d == 0) { s_m[wave][row] = M; s_l[wave][row] = L; }
                }
                __syncthreads();
                for (int i = 2 * tid; i < rows * DP; i += 2 * THREADS) {
                    float M, L, x, y;
                    join(i / DP, i % DP, &M, &L, &x, &y);
                    finish(i / DP, i % DP, M, L, x, y);
                }
            }
        }
        u += to - from;
        if (u - first >= nu * per_seq) { first += nu * per_seq; ++seq; }
    }
}

// weight = decay * weight + the sum over the query heads of a key head of e^(s - lse), four slots a thread.
__global__ __launch_bounds__(256) void weight_kernel(const AttendArgs a)
{
    const int seq = blockIdx.z, h = blockIdx.y, slot = (blockIdx.x * 256 + threadIdx.x) * 4, len = clamp_length(a.c.lengths[seq], a.c.capacity);
    if (slot >= len) return;
    const long q_head = (long)seq * a.j.q.heads + h * a.group;
    const float* s = a.scores + q_head * a.pitch + slot;
    float* to = a.c.weight + ((long)seq * a.c.heads + h) * a.c.capacity + slot;
    f32x4 sum = f32x4{0, 0, 0, 0}, w = *reinterpret_cast<const f32x4*>(to);
    for (int g = 0; g < a.group; ++g) {
        const float z = a.lse[q_head + g];
        const f32x4 x = *reinterpret_cast<const f32x4*>(s + (long)g * a.pitch);
        if (z != -__builtin_inff())
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += exp_of(x[i] - z);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = slot + i < len ? w[i] * a.j.decay + sum[i] : w[i];
    *reinterpret_cast<f32x4*>(to) = w;
}

}  // namespace

bool attend_fits(const Cache& c, int q_heads)
{
    const unsigned long long blocks = (unsigned)(q_heads / c.heads + ROWS - 1) / ROWS, units = (unsigned)(c.capacity + UNIT - 1) / UNIT;
    return (unsigned long long)c.seqs * c.heads * blocks * units < (1ull << 31);
}

hipError_t launch_attend(const AttendJob& j, const Cache& c, hipStream_t st)
{
    const ScratchPlan plan = scratch_plan(c, j.q.heads);
    AttendArgs a;
    a.j = j;
    a.c = c;
    a.group = j.q.heads / c.heads;
    a.blocks = (a.group + ROWS - 1) / ROWS;
    const int size = c.bf16 ? 2 : 4, align = 16 / size;
    a.q_aligned = (uintptr_t)j.q.data % 16 == 0 && j.q.token % align == 0 && j.q.head % align == 0;
    a.counters = reinterpret_cast<int*>(c.scratch) + ATTEND_COUNTERS;
    a.parts = reinterpret_cast<float*>(c.scratch + plan.parts);
    a.lse = reinterpret_cast<float*>(c.scratch + plan.lse);
    a.scores = j.accumulate ? reinterpret_cast<float*>(c.scratch + plan.scores) : nullptr;
    a.pitch = c.capacity;
    const int dp = c.dim <= 64 ? 64 : (c.dim <= 128 ? 128 : 256);
    // one workgroup a compute unit, no more than there can be units
    const long most = (long)c.seqs * c.heads * a.blocks * ((c.capacity + UNIT - 1) / UNIT);
    const long want = device_units();
    const int groups = (int)(most < want ? most : (want < MAX_GROUPS ? want : MAX_GROUPS));
#define CB_ATTEND(type, d) hipLaunchKernelGGL((attend_kernel<type, d>), dim3(groups), dim3(Tile<type, d>::WAVES * 64), 0, st, a)
    if (c.bf16) {
        if (dp == 64) CB_ATTEND(uint16_t, 64);
        else if (dp == 128) CB_ATTEND(uint16_t, 128);
        else CB_ATTEND(uint16_t, 256);
    } else {
        if (dp == 64) CB_ATTEND(float, 64);
        else if (dp == 128) CB_ATTEND(float, 128);
        else CB_ATTEND(float, 256);
    }
#undef CB_ATTEND
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !j.accumulate) return e;
    hipLaunchKernelGGL(weight_kernel, dim3((c.capacity + 1023) / 1024, c.heads, c.seqs), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace cb
