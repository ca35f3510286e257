// Attention of one new token per sequence over a paged key-value cache.
//
// For each sequence and key head: s_j = scale q.k_j for the query heads that read the key head, the softmax over the
// cached tokens j, and the weighted sum of the v_j.  Keys and values are read once, so memory bounds it: 4 * dim * heads operations for
// 2 * dim * heads / group values (200 003 tokens of 8 key heads, 128 values in bfloat16: 131 us, 6.3 TB/s, where plain reads reach 7.2; 6.6 over
// 32 x 8 192 tokens).  More than 16 query heads a key head are blocks of 16, and every block reads the keys and values again.
// One pass: every wavefront takes tiles of consecutive tokens and keeps, for up to 16 query heads, the running maximum m, the sum l of e^(s - m) and the sum o of e^(s - m) v (times a power of two, see Tiles::bits); a tile with a larger maximum scales l and o by e^(m - m').
// Parts of a sequence (wavefronts of a workgroup, then workgroups) are joined the same way.
//
// Layout.  S^T = K Q^T and O^T = V^T P^T on the matrix cores, 16 query heads as columns.  A lane's column is its query head (lane & 15) in both, so
// that m and l live in the lane that needs them, and what S^T leaves in a lane -- the scores of tokens 4 * (lane >> 4) + r -- is
// what P^T wants there, if the tokens of a tile are numbered to suit; no value changes lanes but for the maximum.  Keys and values come
// from memory into registers as the matrix cores take them, whole rows by neighbouring lanes.
//
// Work is split over the length, whatever the lengths, which the kernel reads itself.  Where there are workgroups enough, every pair (sequence,
// key head, block of query heads) has its own, more of them the longer it is; where there are not, the tiles of all pairs, in order, are dealt to
// the workgroups in equal runs.  A run is dealt to the wavefronts in the same way.  A wavefront goes through its part by itself: what it has
// whole it finishes, and what begins or ends in the middle of something waits in LDS until all wavefronts are through.  What
// begins or ends in the middle of something for the workgroup goes to the scratch buffer, and the workgroup that comes last of those that
// share it joins the parts, in order.
#include <type_traits>

#include "cb_tokens.h"

namespace cb {

namespace {

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896340736f, LOG2E_REST = (float)(1.44269504088896340736 - (double)LOG2E), LN2 = 0.69314718055994530942f;
constexpr float LOWEST = -3.402823466e38f;       // of a maximum, so that nothing is subtracted from minus infinity
constexpr int ROWS = ATTEND_ROWS;
// Tiles of a wavefront that are worth a workgroup of their own: a part more costs its way through memory and the join.  (Measured for five sequences of
// 1 - 9 001 tokens, float32 and 80 values a head: 25.8 us with 1, 22.6 with 2, 28.4 with 4.  Other head sizes and bfloat16 were not.)
constexpr int SPLIT_TILES = 2;

struct AttendArgs {
    AttendJob j;
    Cache c;
    int group, blocks;             // query heads of a key head, blocks of ROWS of them
    int q_aligned, out_aligned;    // to 16 bytes
    int* counters;
    float *parts, *scores;
    float2* sums;                  // of (sequence, query head): the maximum of the scores, 1 / the sum of e^(s - maximum) (0: there is none)
    int pitch;                     // of a query head's scores
};

// e^x for the difference x of two scores, which is exact or nearly so; scores times log2 e would be rounded at their own size.  What the product is
// rounded by, and what log2 e is, come in as a factor 1 + rest: without it e^-80 would be off by 2e-6 of itself (and five sequences of 1 - 9 001 tokens in
// float32 take 22.6 us instead of 23.5, 24 in bfloat16 57.9 instead of 58.6).
__device__ __forceinline__ float exp_of(float x)
{
    const float y = x * LOG2E, rest = __builtin_fmaf(x, LOG2E_REST, __builtin_fmaf(x, LOG2E, -y)), e = __builtin_amdgcn_exp2f(y);
    return e == 0.0f ? 0.0f : __builtin_fmaf(e, rest * LN2, e);      // (minus infinity leaves a rest that is not a number)
}

// 2^e, e from -126 to 127.
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// Two bfloat16 values, the largest finite one of its sign in the place of one that is not finite.  (As integers positive numbers ascend, and so do
// negative ones that are taken as unsigned.)
__device__ __forceinline__ uint32_t finite_halves(uint32_t w)
{
    const i16x2 x = __builtin_elementwise_min(__builtin_bit_cast(i16x2, w), i16x2{0x7F7F, 0x7F7F});
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, x), u16x2{0xFF7F, 0xFF7F}));
}

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

// The tiles of the sequences in order.  All of it is the same for every lane of a wavefront.
struct Tiles {
    const int32_t* lengths;
    int seqs, capacity, per_seq;       // per_seq: (key head, block) pairs of a sequence
    int tokens, enough;                // of a tile; tiles of a pair that keep a workgroup busy
    __device__ int of(int len) const { return len > tokens ? (len + tokens - 1) / tokens : 1; }
    // workgroups that a pair of n tiles is worth: more than one where each has `enough`
    __device__ int worth(int n) const { return n < 2 * enough ? 1 : n / enough; }
    // Sums of e^(s - m) v over a pair of n tiles are kept times 2^-bits, the number of its tokens at least twice: they are a part of a weighted mean
    // then, and no larger than the values, where they could pass float32's range.  (What is lost is below 2^-126 * 2^bits: 1e-32 for
    // 200 000 tokens.)
    __device__ int bits(int n) const { return 33 - __builtin_clz(n) + (31 - __builtin_clz(tokens)); }
    __device__ void total(unsigned* tiles, unsigned* groups) const
    {
        const int lane = threadIdx.x & 63;
        int sum = 0, all = 0;
        for (int s = lane; s < seqs; s += 64) {
            const int n = of(clamp_length(lengths[s], capacity));
            sum += n;
            all += worth(n);
        }
        *tiles = (unsigned)__builtin_amdgcn_readlane(wave_scan(sum), 63) * per_seq;
        *groups = (unsigned)__builtin_amdgcn_readlane(wave_scan(all), 63) * per_seq;
    }
    // the sequence that tile (by_worth: workgroup) u belongs to, and its first one
    __device__ int find(int u, bool by_worth, int* first) const
    {
        const int lane = threadIdx.x & 63;
        int before = 0;
        for (int s0 = 0; s0 < seqs; s0 += 64) {
            const int n = s0 + lane < seqs ? of(clamp_length(lengths[s0 + lane], capacity)) : 0;
            const int sum = wave_scan((by_worth && n ? worth(n) : n) * per_seq);
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

// n tiles dealt to w: the first n % w get one more than the others.
struct Deal {
    unsigned each, more;
    __device__ Deal(unsigned n, unsigned w) : each(n / w), more(n % w) {}
    __device__ unsigned first(unsigned g) const { return g * each + (g < more ? g : more); }
    __device__ unsigned owner(unsigned u) const      // (each is not 0)
    {
        const unsigned big = more * (each + 1);
        return u < big ? u / (each + 1) : more + (u - big) / each;
    }
};

// How a type's tiles look.  PE: consecutive values of a row that a lane takes of V, NP such pieces 16 * PE apart.
template <typename T, int DP> struct Tile;
template <int DP> struct Tile<uint16_t, DP> {
    static constexpr int WAVES = DP == 256 ? 4 : (DP == 64 ? 16 : 8);
    static constexpr int TOKENS = 32, PE = DP == 64 ? 4 : 8, NP = DP / (16 * PE);
    static constexpr int KSTEPS = DP / 32;       // of S^T: 32 values of a head a step
};
template <int DP> struct Tile<float, DP> {
    static constexpr int WAVES = DP == 256 ? 4 : (DP == 64 ? 16 : 8);
    static constexpr int TOKENS = 16, PE = 4, NP = DP / (16 * PE);
    static constexpr int KSTEPS = DP / 16;       // four steps of 4 values
};

// A wavefront's pages: lane x has that of its sub-tile x (16 tokens) of the next 64.
template <int SUB> __device__ __forceinline__ int load_pages(const int32_t* table, int shift, int n_pages, int tile, int step, int len)
{
    const int lane = threadIdx.x & 63, tok = ((tile + lane / SUB * step) * SUB + lane % SUB) * 16;
    int page = -1;
    if (tok < len) page = table[tok >> shift];
    return (unsigned)page < (unsigned)n_pages ? page : -1;
}

// Rows of a page through a buffer descriptor that ends with the last token: what lies behind it reads as zero, without a branch, and lanes
// that have no value of a row ask for an offset that is always behind it.  Values are read once: around the caches.
constexpr int NOWHERE = 0x40000000;
template <int BYTES> __device__ __forceinline__ auto load_row(__amdgpu_buffer_rsrc_t rows, int offset)
{
    constexpr int AROUND = 2;          // non-temporal
    if constexpr (BYTES == 16) return __builtin_amdgcn_raw_buffer_load_b128(rows, offset, 0, AROUND);
    else return __builtin_amdgcn_raw_buffer_load_b64(rows, offset, 0, AROUND);
}

template <typename T, int DP>
__global__ __launch_bounds__((Tile<T, DP>::WAVES * 64)) void attend_kernel(const AttendArgs a)
{
    constexpr bool HALF = sizeof(T) == 2;
    typedef Tile<T, DP> TL;
    constexpr int WAVES = TL::WAVES, THREADS = WAVES * 64, SUB = TL::TOKENS / 16, NP = TL::NP, PE = TL::PE, KSTEPS = TL::KSTEPS;
    constexpr int DW = PE * (int)sizeof(T) / 4;                        // 32-bit words of a piece
    typedef uint32_t piece_t __attribute__((ext_vector_type(DW)));
    typedef uint32_t key_t __attribute__((ext_vector_type(4)));
    // a wavefront's two parts: of what begins before its run, and of what goes on behind it
    __shared__ __align__(16) float s_o[2 * WAVES][ROWS][DP + 4];
    __shared__ float s_m[2 * WAVES][ROWS], s_l[2 * WAVES][ROWS];
    __shared__ int4 s_part[2 * WAVES];                                 // its pair's first tile (-1: no part), sequence, number, tiles
    __shared__ int s_last[2];

    const Cache& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, quad = lane >> 4;
    const int D = c.dim, per_seq = c.heads * a.blocks;
    const Tiles tiles{c.lengths, c.seqs, c.capacity, per_seq, TL::TOKENS, SPLIT_TILES * WAVES};
    unsigned total, groups;
    tiles.total(&total, &groups);
    const bool own_group = groups <= gridDim.x;                        // of a pair
    groups = own_group ? groups : gridDim.x;
    if (blockIdx.x >= groups) return;
    const Deal deal(total, groups);
    // this workgroup's run of tiles (with groups of their own counted from the sequence's first), the sequence that it begins in and that one's first tile
    int run, run_end, seq, first = 0, part = 0, parts = 1;
    if (own_group) {
        int first_group;
        seq = tiles.find(blockIdx.x, true, &first_group);
        if (seq >= c.seqs) return;
        const int n = tiles.of(clamp_length(c.lengths[seq], c.capacity));
        parts = tiles.worth(n);
        const int at = (int)blockIdx.x - first_group, pair = (unsigned)at / (unsigned)parts;
        part = at - pair * parts;
        const Deal split(n, parts);
        run = pair * n + split.first(part);
        run_end = pair * n + split.first(part + 1);
    } else {
        run = deal.first(blockIdx.x);
        run_end = deal.first(blockIdx.x + 1);
    }
    const Deal own(run_end - run, WAVES);
    int u = run + own.first(wave);
    int end = run + own.first(wave + 1);
    int step = 1;
    if (lane < 2) s_part[2 * wave + lane].x = -1;

    // A run is worked through a pair (sequence, head, block) at a time: those of its tiles that fall into one.
    struct Stretch {
        int seq, first, len, n, pair, from, to, h, row0, rows;        // first: tile of the sequence's first pair; n: tiles of a pair
        float down;                                                   // 2^-bits
    };
    auto stretch = [&](int seq, int first) {
        Stretch x;
        x.seq = seq;
        x.first = first;
        x.len = clamp_length(c.lengths[seq], c.capacity);
        x.n = tiles.of(x.len);
        x.down = power(-tiles.bits(x.n));
        x.pair = (unsigned)(u - first) / (unsigned)x.n;
        x.from = u - first - x.pair * x.n;
        x.to = x.n - x.from < end - u ? x.n : x.from + (end - u);
        x.h = (unsigned)x.pair / (unsigned)a.blocks;
        x.row0 = (x.pair - x.h * a.blocks) * ROWS;
        x.rows = a.group - x.row0 < ROWS ? a.group - x.row0 : ROWS;
        return x;
    };
    // tile: where its sub-tiles' rows are (in values), how many tokens they hold
    struct Where { long at[SUB]; int left[SUB]; };
    key_t q[KSTEPS], k[SUB][KSTEPS];
    piece_t v[SUB][4][NP];
    int pages = -1, ahead = -1, used = 0;                      // of the tiles that come
    auto find = [&](const Stretch& x, int tile) {
        Where w;
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            const int tok = tile * TL::TOKENS + 16 * s, page = __builtin_amdgcn_readlane(pages, used * SUB + s);
            w.left[s] = page >= 0 ? (x.len - tok < 16 ? x.len - tok : 16) : 0;
            w.at[s] = page >= 0 ? ((((long)page * c.heads + x.h) << c.page_shift) + (tok & ((1 << c.page_shift) - 1))) * D : 0;
        }
        return w;
    };
    auto rows_of = [&](const void* pages, const Where& w, int s) {
        return __builtin_amdgcn_make_buffer_rsrc((char*)pages + w.at[s] * (long)sizeof(T), 0, w.left[s] * D * (int)sizeof(T), 0x00027000);
    };
    auto load_k = [&](const Where& w) {
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            const __amdgpu_buffer_rsrc_t rows = rows_of(c.k, w, s);
#pragma unroll
            for (int i = 0; i < KSTEPS; ++i) {
                const int d = (4 * i + quad) * (16 / (int)sizeof(T));
                k[s][i] = load_row<16>(rows, d < D ? (l16 * D + d) * (int)sizeof(T) : NOWHERE);
            }
        }
    };
    auto load_v = [&](const Where& w) {
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            const __amdgpu_buffer_rsrc_t rows = rows_of(c.v, w, s);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const int d = (16 * p + l16) * PE;
                    v[s][r][p] = load_row<PE * (int)sizeof(T)>(rows, d < D ? ((4 * quad + r) * D + d) * (int)sizeof(T) : NOWHERE);
                }
        }
    };
    auto load_q = [&](const Stretch& x) {                      // head l16, values 32 * i + 8 * quad .. (or 16 * i + 4 * quad ..)
        const T* src = (const T*)a.j.q.data + (long)x.seq * a.j.q.token + (long)(x.h * a.group + x.row0 + l16) * a.j.q.head;
        constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < KSTEPS; ++i) {
            const int d = (4 * i + quad) * E;
            q[i] = key_t(0);
            if (l16 < x.rows && d < D) {
                if (a.q_aligned) q[i] = *reinterpret_cast<const key_t*>(src + d);
                else {
                    T e[E];
#pragma unroll
                    for (int y = 0; y < E; ++y) e[y] = src[d + y];
                    __builtin_memcpy(&q[i], e, 16);
                }
            }
        }
    };

    auto put_sums = [&](long at, float M, float L) {
        if (a.j.lse) a.j.lse[at] = L == 0.0f ? -__builtin_inff() : M + logf(L);
        if (a.scores) a.sums[at] = make_float2(M, L == 0.0f ? 0.0f : 1.0f / L);
    };
    // row, values d and d + 1 of a pair's result: x and y over L, times 2^bits
    auto store_pair = [&](int seq, int head, int d, float x, float y) {
        if (d >= D) return;
        T* out = (T*)a.j.out.data + (long)seq * a.j.out.token + (long)head * a.j.out.head + d;
        T e0, e1;
        narrow(x, e0);
        narrow(y, e1);
        out[0] = e0;
        out[1] = e1;
    };
    auto finish = [&](int seq, int head, int d, float M, float L, float up, float x, float y) {
        const float inv = L == 0.0f ? 0.0f : up / L;
        store_pair(seq, head, d, x * inv, y * inv);
        if (d == 0) put_sums((long)seq * a.j.q.heads + head, M, L);
    };

    // The tiles in order, those of the run's pairs behind each other: while one is computed the next one comes, its keys while this one's
    // weights are made, its values while the next one's scores are.
    Stretch x, y;                                              // of this tile, of the next one
    int t = 0, ty = 0;                                         // the tiles
    bool here = false, more = u < end;                         // there is one
    Where w, wy;
    float m = LOWEST, l = 0.0f;
    f32x4 o[NP * PE];
#pragma unroll
    for (int i = 0; i < NP * PE; ++i) o[i] = f32x4{0, 0, 0, 0};
    if (more) {
        if (!own_group) seq = tiles.find(u, false, &first);
        // a run within one pair: the wavefronts take its tiles in turn, so that they read one stretch of memory together
        const int n = seq < c.seqs ? tiles.of(clamp_length(c.lengths[seq], c.capacity)) : 1;
        if (run_end - run >= WAVES && run >= first && (unsigned)(run - first) / (unsigned)n == (unsigned)(run_end - 1 - first) / (unsigned)n) {
            step = WAVES;
            u = run;
            end = run_end;
        }
        more = seq < c.seqs;
    }
    bool fresh = true;                                         // the next tile begins a stretch
    for (;;) {
        f32x4 sc[SUB];
        if (here) {
            // scores of tokens 16 * s + 4 * quad + r for query head l16
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                sc[s] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < KSTEPS; ++i) {
                    if constexpr (HALF)
                        sc[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[s][i]), __builtin_bit_cast(bf16x8, q[i]), sc[s], 0, 0, 0);
                    else {
                        const f32x4 ka = __builtin_bit_cast(f32x4, k[s][i]), qa = __builtin_bit_cast(f32x4, q[i]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[s] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka[e], qa[e], sc[s], 0, 0, 0);
                    }
                }
            }
        }
        // the next tile: of this stretch, or the first one of the next
        if (more) {
            if (fresh) {
                y = stretch(seq, first);
                ty = y.from + (step > 1 ? wave : 0);
                used = 0;
                pages = load_pages<SUB>(c.table + (long)y.seq * c.max_pages, c.page_shift, c.n_pages, ty, step, y.len);
                load_q(y);
            } else if (++used == 64 / SUB) {
                used = 0;
                pages = ahead;
            }
            if (used == 0 && ty + 64 / SUB * step < y.to)
                ahead = load_pages<SUB>(c.table + (long)y.seq * c.max_pages, c.page_shift, c.n_pages, ty + 64 / SUB * step, step, y.len);
            wy = find(y, ty);
            load_k(wy);
        }
        if (here) {
            float top = LOWEST;
#pragma unroll
            for (int s = 0; s < SUB; ++s)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float y = sc[s][r] * a.j.scale;
                    if (a.j.softcap > 0.0f) y = a.j.softcap * tanhf(y / a.j.softcap);
                    y = 4 * quad + r < w.left[s] ? y : -__builtin_inff();
                    sc[s][r] = y;
                    top = fmaxf(top, y);
                }
            if (a.scores && l16 < x.rows) {
                float* to_scores = a.scores + ((long)x.seq * a.j.q.heads + x.h * a.group + x.row0 + l16) * a.pitch + t * TL::TOKENS + 4 * quad;
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
                    p[s][r] *= x.down;
                }
            if constexpr (HALF) {
                // P in three bfloat16 terms of 8 significant bits each, cut off and not rounded: they hold all of a float32's 24 bits, so that P is
                // no less exact than in float32 (two terms put the sums off by 2^-18 of the values; 200 003 tokens take 133 us instead of 132)
                uint32_t cut[3][8];
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    float rest = p[x / 4][x % 4];
#pragma unroll
                    for (int y = 0; y < 3; ++y) {
                        cut[y][x] = __float_as_uint(rest) & 0xFFFF0000u;
                        rest -= __uint_as_float(cut[y][x]);
                    }
                }
                bf16x8 terms[3];
#pragma unroll
                for (int y = 0; y < 3; ++y) {
                    uint32_t w[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) w[x] = __builtin_amdgcn_perm(cut[y][2 * x + 1], cut[y][2 * x], 0x07060302u);
                    terms[y] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
                }
                // (The lower terms may be zero where P is not, and zero times infinity is not a number: they meet finite values alone.)
                auto add_values = [&](auto clamp) {
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
                            f32x4& to = o[pc * PE + e];
                            to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3])), terms[0], to, 0, 0, 0);
                            if constexpr (clamp.value)
#pragma unroll
                                for (int x = 0; x < 4; ++x) w[x] = finite_halves(w[x]);
#pragma unroll
                            for (int y = 1; y < 3; ++y)
                                to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3])), terms[y], to, 0, 0, 0);
                        }
                };
                // Two instructions a word, or a question for 64 lanes and a branch, which takes 60 registers more.  Rows of 65 - 128 values have them: 200 003
                // tokens 130.6 us with the branch, 135.6 without, 24 streams 48.4 and 49.2.  Up to 64 values some would wait in scratch memory (132.5 and 77.2 us, 54.6
                // and 36.9), above 128 there is no difference (252.0 and 252.0, 83.1 and 82.8).
                if constexpr (DP == 128) {
                    u16x2 size = {0, 0};                       // the largest exponents, of both halves of the words
#pragma unroll
                    for (int s = 0; s < SUB; ++s)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int pc = 0; pc < NP; ++pc)
#pragma unroll
                                for (int x = 0; x < DW; ++x) size = __builtin_elementwise_max(size, __builtin_bit_cast(u16x2, v[s][r][pc][x] & 0x7F807F80u));
                    if (__ballot(size[0] == 0x7F80 || size[1] == 0x7F80)) add_values(std::true_type());
                    else add_values(std::false_type());
                } else add_values(std::true_type());
            } else {
#pragma unroll
                for (int pc = 0; pc < NP; ++pc)
#pragma unroll
                    for (int e = 0; e < PE; ++e)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            o[pc * PE + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[0][r][pc][e]), p[0][r], o[pc * PE + e], 0, 0, 0);
            }
        }
        if (more) load_v(wy);
        if (here && t + step >= x.to) {
            // the pair is through, as far as this wavefront has to do with it
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            // lane has o of query head l16, values (16 * p + 4 * quad + r) * PE + e: runs of 4 * PE values
            if (x.from == 0 && x.to == x.n && step == 1) {
                const int head = x.h * a.group + x.row0 + l16;
                const float inv = l == 0.0f ? 0.0f : power(tiles.bits(x.n)) / l;
                if (l16 < x.rows) {
                    T* out = (T*)a.j.out.data + (long)x.seq * a.j.out.token + (long)head * a.j.out.head;
                    constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
                    for (int p = 0; p < NP; ++p)
#pragma unroll
                        for (int i = 0; i < 4 * PE / E; ++i) {
                            const int d = (16 * p + 4 * quad) * PE + i * E;
                            T e[E];
#pragma unroll
                            for (int z = 0; z < E; ++z) narrow(o[p * PE + (i * E + z) % PE][(i * E + z) / PE] * inv, e[z]);
                            if (d < D) {
                                if (a.out_aligned) {
                                    key_t word;
                                    __builtin_memcpy(&word, e, 16);
                                    *reinterpret_cast<key_t*>(out + d) = word;
                                } else
#pragma unroll
                                    for (int z = 0; z < E; ++z) out[d + z] = e[z];
                            }
                        }
                    if (quad == 0) put_sums((long)x.seq * a.j.q.heads + head, m, l);
                }
            } else {
                const int slot = 2 * wave + (x.from == 0 && (step == 1 || wave == 0) ? 1 : 0);
                if (quad == 0) { s_m[slot][l16] = m; s_l[slot][l16] = l; }
                if (l16 < x.rows) {
#pragma unroll
                    for (int p = 0; p < NP; ++p)
#pragma unroll
                        for (int i = 0; i < PE; ++i) {
                            f32x4 e;
#pragma unroll
                            for (int z = 0; z < 4; ++z) e[z] = o[p * PE + (4 * i + z) % PE][(4 * i + z) / PE];
                            *reinterpret_cast<f32x4*>(&s_o[slot][l16][(16 * p + 4 * quad) * PE + 4 * i]) = e;
                        }
                }
                if (lane == 0) s_part[slot] = make_int4(x.first + x.pair * x.n, x.seq, x.pair, x.n);
            }
            m = LOWEST;
            l = 0.0f;
#pragma unroll
            for (int i = 0; i < NP * PE; ++i) o[i] = f32x4{0, 0, 0, 0};
        }
        here = more;
        if (!here) break;
        if (fresh) x = y;
        t = ty;
        w = wy;
        // and what comes behind that one
        ty += step;
        fresh = ty >= y.to;
        if (fresh) {
            u += y.to - y.from;
            if (u - y.first >= y.n * per_seq) { ++seq; first += y.n * per_seq; }
            more = u < end && seq < c.seqs;
        }
    }
    __syncthreads();

    // The parts of a pair: the first one a part that goes on behind its wavefront's run (or the workgroup's first part, of what begins before its
    // run), the others the first parts of the wavefronts behind.  Wavefronts without tiles are behind all others.
    const int4 of_slot = s_part[lane & (2 * WAVES - 1)];       // a slot a lane
    struct Chain { int slot, wave, parts, seq, first, n, head0, rows; };
    auto chain = [&](int slot) {
        Chain x;
        x.slot = slot;
        x.first = __builtin_amdgcn_readlane(of_slot.x, slot);
        x.seq = __builtin_amdgcn_readlane(of_slot.y, slot);
        const int pair = __builtin_amdgcn_readlane(of_slot.z, slot);
        x.n = __builtin_amdgcn_readlane(of_slot.w, slot);
        x.wave = slot >> 1;
        // the run of wavefronts behind whose first parts are of the same pair
        const unsigned long long others = ~__ballot((lane & 1) == 0 && lane < 2 * WAVES && of_slot.x == x.first) & 0x5555555555555555ull;
        x.parts = (__builtin_ctzll(others >> (2 * x.wave + 2) | 1ull << (2 * (WAVES - 1 - x.wave))) >> 1) + 1;
        const int h = (unsigned)pair / (unsigned)a.blocks, row0 = (pair - h * a.blocks) * ROWS;
        x.head0 = h * a.group + row0;
        x.rows = a.group - row0 < ROWS ? a.group - row0 : ROWS;
        return x;
    };
    // slot s0 and the first slots of the wavefronts behind `rest`, `parts` in all: row, values d and d + 1
    auto join = [&](int s0, int rest, int parts, int row, int d, float* M, float* L, float* x, float* y) {
        float mp[WAVES], lp[WAVES];
        float2 v[WAVES];
        *M = LOWEST;
#pragma unroll
        for (int p = 0; p < WAVES; ++p) {
            mp[p] = LOWEST;
            lp[p] = 0.0f;
            v[p] = make_float2(0.0f, 0.0f);
            if (p < parts) {
                const int s = p == 0 ? s0 : 2 * (rest + p);
                mp[p] = s_m[s][row];
                lp[p] = s_l[s][row];
                v[p] = *reinterpret_cast<const float2*>(&s_o[s][row][d]);
            }
            *M = fmaxf(*M, mp[p]);
        }
        *L = *x = *y = 0.0f;
#pragma unroll
        for (int p = 0; p < WAVES; ++p) {
            const float f = exp_of(mp[p] - *M);
            *L += f * lp[p];
            *x += f * v[p].x;
            *y += f * v[p].y;
        }
    };
    bool mine[2] = {false, false};                             // parts of this workgroup that others have to do with
    // (a part that begins before its wavefront's run belongs to the chain of an earlier one, but for the workgroup's first)
    const unsigned long long heads = __ballot(lane < 2 * WAVES && of_slot.x >= 0 && (lane == 0 || (lane & 1)));
    for (unsigned long long rest = heads; rest; rest &= rest - 1) {
        const Chain x = chain(__builtin_ctzll(rest));
        const bool whole = x.first >= run && x.first + x.n <= run_end;
        const int w = x.first < run ? 0 : 1;
        float* to = a.parts + (2L * blockIdx.x + w) * part_floats<DP>();
        for (int i = 2 * tid; i < x.rows * DP; i += 2 * THREADS) {
            const int row = i / DP, d = i % DP;
            float M, L, y, z;
            join(x.slot, x.wave, x.parts, row, d, &M, &L, &y, &z);
            if (whole) finish(x.seq, x.head0 + row, d, M, L, power(tiles.bits(x.n)), y, z);
            else {
                put(to + 2 * ROWS + i, y, z);
                if (d == 0) put(to + 2 * row, M, L);
            }
        }
        if (!whole) mine[w] = true;
    }
    if (!mine[0] && !mine[1]) return;
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0): this wavefront's stores are where every compute unit sees them
    __syncthreads();
    // the workgroups that share a pair count themselves at its first one's counter; that one has no other pair that goes on behind it
    int slots[2] = {0, 0};
    unsigned w0[2] = {0, 0}, w1[2] = {0, 0};
    for (int w = 0; w < 2; ++w)
        if (mine[w]) {
            slots[w] = w == 0 ? 0 : 63 - __builtin_clzll(heads);       // the workgroup's first part, or the last one that goes on
            const unsigned u0 = __builtin_amdgcn_readlane(of_slot.x, slots[w]);
            w0[w] = own_group ? blockIdx.x - part : deal.owner(u0);
            w1[w] = own_group ? w0[w] + parts - 1 : deal.owner(u0 + __builtin_amdgcn_readlane(of_slot.w, slots[w]) - 1);
            if (tid == w) {
                int* counter = a.counters + w0[w];
                s_last[w] = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)(w1[w] - w0[w]);
                if (s_last[w]) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
    __syncthreads();
    for (int w = 0; w < 2; ++w) {
        if (!mine[w] || !s_last[w]) continue;
        const Chain x = chain(slots[w]);
        const int rows = x.rows;
        // the weight of every part, a query head a wavefront at a time (LDS is free but for what the parts are of, which is in registers)
        const int count = (int)(w1[w] - w0[w]) + 1;
        float* s_weight = &s_o[0][0][0];                       // rows x parts
        float* s_sum = &s_o[WAVES][0][0];
        static_assert(WAVES * ROWS * (DP + 4) >= ROWS * MAX_GROUPS, "room for the weights of all parts");
        auto part_of = [&](int p) { return a.parts + (2L * (w0[w] + p) + (p == 0 ? 1 : 0)) * part_floats<DP>(); };
#pragma unroll 1
        for (int row = wave; row < rows; row += WAVES) {
            float M = LOWEST, L = 0.0f;
#pragma unroll 1
            for (int p = lane; p < count; p += 64) {
                const float2 ml = get(part_of(p) + 2 * row);
                s_weight[row * count + p] = ml.x;
                s_sum[row * count + p] = ml.y;
                M = fmaxf(M, ml.x);
            }
            M = wave_max(M);
#pragma unroll 1
            for (int p = lane; p < count; p += 64) L += exp_of(s_weight[row * count + p] - M) * s_sum[row * count + p];
            L = wave_sum(L);
            const float inv = L == 0.0f ? 0.0f : power(tiles.bits(x.n)) / L;
#pragma unroll 1
            for (int p = lane; p < count; p += 64) s_weight[row * count + p] = exp_of(s_weight[row * count + p] - M) * inv;
            if (lane == 0) put_sums((long)x.seq * a.j.q.heads + x.head0 + row, M, L);
        }
        __syncthreads();
        // the sum over the parts, two values a thread: a team of threads for all of them takes every teams-th part, in order
        const int pairs = rows * DP / 2, teams = THREADS / pairs > 1 ? THREADS / pairs : 1, team = tid / pairs;
#pragma unroll 1
        for (int i = teams > 1 ? tid - team * pairs : tid; i < pairs && team < (teams > 1 ? teams : WAVES * 64); i += teams > 1 ? pairs : THREADS) {
            const int row = 2 * i / DP, d = 2 * i % DP;
            float y = 0.0f, z = 0.0f;
#pragma unroll 1
            for (int p = teams > 1 ? team : 0; p < count; p += 8 * teams) {
                float2 v[8];
#pragma unroll
                for (int n = 0; n < 8; ++n) v[n] = get(part_of(p + n * teams < count ? p + n * teams : p) + 2 * ROWS + 2 * i);
#pragma unroll
                for (int n = 0; n < 8; ++n)
                    if (p + n * teams < count) {
                        const float f = s_weight[row * count + p + n * teams];
                        y += f * v[n].x;
                        z += f * v[n].y;
                    }
            }
            if (teams > 1) *reinterpret_cast<float2*>(s_sum + 2 * (team * pairs + i)) = make_float2(y, z);
            else store_pair(x.seq, x.head0 + row, d, y, z);
        }
        if (teams > 1) {
            __syncthreads();
            if (team == 0) {
                float y = 0.0f, z = 0.0f;
#pragma unroll 1
                for (int n = 0; n < teams; ++n) {
                    const float2 v = *reinterpret_cast<const float2*>(s_sum + 2 * (n * pairs + tid));
                    y += v.x;
                    z += v.y;
                }
                store_pair(x.seq, x.head0 + 2 * tid / DP, 2 * tid % DP, y, z);
            }
        }
        __syncthreads();
    }
}

// weight = decay * weight + the sum over the query heads of a key head of e^(s - m) / l, four slots a thread.  (Not e^(s - lse): the logarithm of l
// would be rounded at the size of m, and be lost altogether beside a large one.)  A launch of its own, since m and l are
// only known when all parts are joined: the scores wait in the scratch buffer (4 bytes a query head where keys and values are 4 * dim;
// 24 sequences of 53 855 tokens in all, 32 query heads: 5 us here, 11 us of the 59 with the scores' way and the launch).
__global__ __launch_bounds__(256) void weight_kernel(const AttendArgs a)
{
    const int seq = blockIdx.z, h = blockIdx.y, slot = (blockIdx.x * 256 + threadIdx.x) * 4, len = clamp_length(a.c.lengths[seq], a.c.capacity);
    if (slot >= len) return;
    if ((unsigned)a.c.table[(long)seq * a.c.max_pages + (slot >> a.c.page_shift)] >= (unsigned)a.c.n_pages) return;      // no page: no token
    const long q_head = (long)seq * a.j.q.heads + h * a.group;
    const float* s = a.scores + q_head * a.pitch + slot;
    float* to = a.c.weight + ((long)seq * a.c.heads + h) * a.c.capacity + slot;
    f32x4 sum = f32x4{0, 0, 0, 0}, w = *reinterpret_cast<const f32x4*>(to);
    for (int g = 0; g < a.group; ++g) {
        const float2 ml = a.sums[q_head + g];
        const f32x4 x = *reinterpret_cast<const f32x4*>(s + (long)g * a.pitch);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += exp_of(x[i] - ml.x) * ml.y;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = slot + i < len ? w[i] * a.j.decay + sum[i] : w[i];
    *reinterpret_cast<f32x4*>(to) = w;
}

}  // namespace

bool attend_fits(const Cache& c, int q_heads)
{
    const unsigned long long blocks = (unsigned)(q_heads / c.heads + ROWS - 1) / ROWS, tiles = (unsigned)c.capacity / 16;
    return (unsigned long long)c.seqs * c.heads * blocks * tiles < (1ull << 31);
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
    a.sums = reinterpret_cast<float2*>(c.scratch + plan.sums);
    a.scores = j.accumulate ? reinterpret_cast<float*>(c.scratch + plan.scores) : nullptr;
    a.pitch = c.capacity;
    const int dp = c.dim <= 64 ? 64 : (c.dim <= 128 ? 128 : 256);
    a.out_aligned = (uintptr_t)j.out.data % 16 == 0 && j.out.token % align == 0 && j.out.head % align == 0;
    // one workgroup a compute unit, no more than there can be tiles
    const long most = (long)c.seqs * c.heads * a.blocks * (c.capacity / (c.bf16 ? 32 : 16) + 1);
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
