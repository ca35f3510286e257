// Norms of heads with their rotation in the same pass, and the gradients of both.
//
// A head x of D values: n = x r, r = (mean x^2 + eps)^-1/2, out = R(n w), where w has a weight for every value and R turns pairs by the token's
// position (cb_rotary.hip).  Backward, with g = R^-1(gradient of out): the gradient of x is r (w g - n mean(w g n)), that of w the sum over tokens and
// heads of g n.  Since mean(w g n) = r mean(w g x), both sums over a head are made in one go.
//
// Heads are independent and read once, so memory bounds it: 2 values' bytes forward, 3 backward.  38 400 tokens x 40 heads of 128 in bfloat16 take 130 us (6.0
// TB/s, reads and writes; a copy around the caches reaches 6.4), the gradients of 19 200 such tokens 113 us (5.2 TB/s, three wavefronts a SIMD: what
// they hold takes all registers for them) and 5 for the sums of the weights'.  A head lies in the registers of 1 - 64 lanes (two
// vectors of 16 bytes a lane, as pairs need them), its sums take a few steps across them.  A wavefront goes through all heads of its tokens by itself: the
// angles, which it makes once, and all that addresses need stay in its registers.  (With a workgroup for a token, its angles in LDS and a division for every head the
// clip took 208 us.)
// A gradient of the weights is summed by persistent workgroups, the queries' in registers, the keys', which are fewer, in LDS; each leaves one row of sums, and a
// second launch adds these up in order, so that results do not vary.  (Both in registers, and the angles too, left room for two wavefronts a SIMD: 125 us in all instead of 118,
// heads of 80 values 116 instead of 96; but of 256 values 219 instead of 226.)  (The next heads' loads before this one's arithmetic: 13 us more.  Queries and keys, and heads that are
// scaled, in code of their own, 24 KB instead of 16: 6 us more.)
#include <climits>
#include <type_traits>

#include "cb_rows.h"

namespace cb {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64, MAX_DIM = 256;
// Mean squares in float32 are exact enough, and their root's inverse is a normal number, between these; what is beyond is scaled by a power of two first.  Backward
// the sum of x times gradients and weights has to stay within float32's range, too: values within 2^-20 .. 2^24 leave it most of that.
constexpr float SMALL = 0x1p-100f, LARGE = 0x1p100f, SMALL_BACK = 0x1p-40f, LARGE_BACK = 0x1p40f;

// How a wavefront's lanes are dealt: 2^lanes_log to a head, of 2^heads_log heads at a time, of as many tokens as are left over.
struct Shape {
    int pieces, lanes_log, heads_log;      // pieces: two vectors each, of a head
    int q_steps, steps;                    // of 2^heads_log heads: the queries', all
    long stretches;                        // of a wavefront's tokens
};

__device__ __forceinline__ float weight_of(const void* w, int bf16, int i)
{
    return bf16 ? widen(((const uint16_t*)w)[i]) : ((const float*)w)[i];
}

// Over the 2^log lanes of a head, the same in each: partners' values are joined in both lanes of a pair.
template <typename F> __device__ __forceinline__ float over_head(float v, int log, F join)
{
    auto from = [](int b) { return __uint_as_float((uint32_t)b); };
    if (log > 0) v = join(v, from(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0xB1, 0xf, 0xf, true)));      // quad_perm 1 0 3 2
    if (log > 1) v = join(v, from(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x4E, 0xf, 0xf, true)));      // quad_perm 2 3 0 1
    if (log > 2) v = join(v, from(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x141, 0xf, 0xf, true)));     // row_half_mirror
    if (log > 3) v = join(v, from(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x140, 0xf, 0xf, true)));     // row_mirror
    if (log > 4) v = join(v, __shfl_xor(v, 16));
    if (log > 5) v = join(v, __shfl_xor(v, 32));
    return v;
}
__device__ __forceinline__ float head_sum(float v, int log) { return over_head(v, log, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float head_max(float v, int log) { return over_head(v, log, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ int exponent(float v) { return (int)(__float_as_uint(v) >> 23 & 255) - 127; }

// Two vectors of a head's pairs, turned by the lane's angles (see turn() of cb_rows.h for how they lie).  Those behind the pairs stay as they are: a turn by
// nothing would make y * 0 of an infinite value.  (A choice and no branch: with one, adjacent pairs in vectors of 8 values take 135 registers, which leaves three wavefronts
// a SIMD instead of four, and 19 200 tokens with 40 heads of 80 in bfloat16 62.6 us instead of 56.2.)
template <int VE, bool ADJACENT> __device__ __forceinline__ void turn_by(const float2 (&at)[VE], bool turns, float (&a)[VE], float (&b)[VE])
{
    auto pair = [&](float2 cs, float& x, float& y) {
        const float u = __builtin_fmaf(x, cs.x, -(y * cs.y)), v = __builtin_fmaf(x, cs.y, y * cs.x);
        x = turns ? u : x;
        y = turns ? v : y;
    };
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        if constexpr (!ADJACENT) pair(at[e], a[e], b[e]);
        else if (e % 2 == 0) {
            pair(at[e / 2], a[e], a[(e + 1) % VE]);
            pair(at[VE / 2 + e / 2], b[e], b[(e + 1) % VE]);
        }
    }
}

// PPL: pieces of a head that a lane has (more than one where single values are taken of heads above 128).  CACHED: loads and stores go through the caches (where they
// do not, all of a head is turned).
template <typename T, int VE, int PPL, bool ADJACENT, bool CACHED, bool BACK>
__global__ __launch_bounds__(THREADS, VE == 8 ? (BACK ? 3 : 4) : 1) void norm_kernel(const NormJob n, const Shape sh)
{
    typedef Vec<T, VE> V;
    typedef typename Word<sizeof(V)>::type W;
    constexpr int BATCH = BACK ? 2 : 3;          // steps that are on their way at once
    extern __shared__ __align__(16) float2 s_dyn[];      // a wavefront's angles; BACK: its sums in the end
    __shared__ __align__(16) float s_w[2][MAX_DIM + 8];       // behind the weights what there is for no value: zero
    const RotaryJob& j = n.r;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), np = j.pairs, dim = j.dim;
    const int log = sh.lanes_log, sub = lane & ((1 << log) - 1), slot = lane >> log, head0 = slot & ((1 << sh.heads_log) - 1), token = slot >> sh.heads_log;
    const int tokens = (64 >> log) >> sh.heads_log, turned = np / VE;
    const float scale = 1.0f / (float)dim;
    float2* s_cs = s_dyn + wave * tokens * np;
    for (int i = tid; i < 2 * dim; i += THREADS) {
        const void* from = i < dim ? n.q_weight : n.k_weight;
        const int d = i < dim ? i : i - dim;
        s_w[i < dim ? 0 : 1][d] = from ? weight_of(from, n.weight_bf16, d) : 0.0f;
    }
    if (tid < 16) s_w[tid / 8][MAX_DIM + tid % 8] = 0.0f;
    __syncthreads();
    // where a lane's pieces lie in a head, the same of every head
    int first[PPL], second[PPL];
    bool turns[PPL], has_a[PPL], has_b[PPL];
#pragma unroll
    for (int p = 0; p < PPL; ++p) {
        const int piece = sub + (p << log);
        turns[p] = piece < turned;
        first[p] = turns[p] && !j.adjacent ? VE * piece : 2 * VE * piece;
        second[p] = turns[p] && !j.adjacent ? np + VE * piece : 2 * VE * piece + VE;
        has_a[p] = piece < sh.pieces;
        has_b[p] = has_a[p] && second[p] < dim;
        if (!has_a[p]) first[p] = MAX_DIM;
        if (!has_b[p]) second[p] = MAX_DIM;
    }
    // BACK: of g n, of all heads that were here (the keys' in LDS, where a lane has a place of its own)
    constexpr int VALUES = PPL * 2 * VE;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    __shared__ __align__(16) f32x4 s_keys[BACK ? VALUES / 4 : 1][BACK ? THREADS : 1];
    float sum[VALUES] = {};
    if constexpr (BACK)
#pragma unroll
        for (int i = 0; i < VALUES / 4; ++i) s_keys[i][tid] = f32x4{0, 0, 0, 0};

    for (long stretch = (long)blockIdx.x * WAVES + wave; stretch < sh.stretches; stretch += (long)gridDim.x * WAVES) {
        const uint32_t tok = (uint32_t)(stretch * tokens) + (uint32_t)token;      // (there are less than 2^31)
        const bool real = tok < j.tokens;
        W x[BATCH][PPL][2], g[BATCH][PPL][2];
        // (by value: a choice between the arguments' addresses would put them all into scratch memory)
        auto head_at = [&](bool q, Heads a, Heads b, int h) {
            return (const T*)(q ? a.data : b.data) + (long)tok * (q ? a.token : b.token) + (long)h * (q ? a.head : b.head);
        };
        auto get = [](bool there, const T* from) {
            W v = W{};
            if (there) v = CACHED ? *reinterpret_cast<const W*>(from) : __builtin_nontemporal_load(reinterpret_cast<const W*>(from));
            return v;
        };
        auto fetch = [&](int base) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int step = base + u;
                if (step >= sh.steps) continue;
                const bool q = step < sh.q_steps;
                const int h = head0 + ((q ? step : step - sh.q_steps) << sh.heads_log);
                const bool there = real && h < (q ? j.q.heads : j.k.heads);
                const T *src = head_at(q, j.q, j.k, h), *gsrc = BACK ? head_at(q, n.q_grad, n.k_grad, h) : nullptr;
#pragma unroll
                for (int p = 0; p < PPL; ++p) {
                    x[u][p][0] = get(there && has_a[p], src + first[p]);
                    x[u][p][1] = get(there && has_b[p], src + second[p]);
                    if constexpr (BACK) {
                        g[u][p][0] = get(there && has_a[p], gsrc + first[p]);
                        g[u][p][1] = get(there && has_b[p], gsrc + second[p]);
                    }
                }
            }
        };
        fetch(0);
        auto angles = [&](int p, float2 (&to)[VE]) {
#pragma unroll
            for (int e = 0; e < VE; ++e) to[e] = turns[p] ? s_cs[token * np + (sub + (p << log)) * VE + e] : make_float2(1.0f, 0.0f);
        };
        float2 at[PPL][VE];                      // (forward: backward there are no registers for them)
        {
            // (the last stretch's angles have been read: a wavefront's accesses of LDS are in order)
            __builtin_amdgcn_wave_barrier();
            for (int i = lane; i < tokens * np; i += 64) {
                const int t = i / np;
                const long y = stretch * tokens + t;
                s_cs[i] = angle_of(j, y < j.tokens ? y : j.tokens - 1, i - t * np);
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            if constexpr (!BACK) {
#pragma unroll
                for (int p = 0; p < PPL; ++p) angles(p, at[p]);
            }
        }
        auto take = [&](int u, int step) {
            const bool side = step >= sh.q_steps;                    // keys
            const int h = head0 + ((side ? step - sh.q_steps : step) << sh.heads_log);
            const bool there = real && h < (side ? j.k.heads : j.q.heads);
            float f[PPL][2][VE], d[PPL][2][VE], w[PPL][2][VE];       // the head; BACK: its gradient, turned back; the weights
#pragma unroll
            for (int p = 0; p < PPL; ++p) {
                const V xa = __builtin_bit_cast(V, x[u][p][0]), xb = __builtin_bit_cast(V, x[u][p][1]);
                V ga = {}, gb = {};
                if constexpr (BACK) { ga = __builtin_bit_cast(V, g[u][p][0]); gb = __builtin_bit_cast(V, g[u][p][1]); }
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    w[p][0][e] = s_w[side][first[p] + e];
                    w[p][1][e] = s_w[side][second[p] + e];
                    f[p][0][e] = widen(xa.e[e]);
                    f[p][1][e] = widen(xb.e[e]);
                    if constexpr (BACK) {
                        d[p][0][e] = widen(ga.e[e]);
                        d[p][1][e] = widen(gb.e[e]);
                    }
                }
                if constexpr (BACK) {
                    angles(p, at[p]);
                    turn_by<VE, ADJACENT>(at[p], !CACHED || turns[p], d[p][0], d[p][1]);
                }
            }
            float mean, dot;
            int down = 0;                                            // f is the head times 2^-down
            // (once, or once more for a head that has been scaled: a loop, since a kernel's instructions come from memory too)
#pragma unroll 1
            for (bool again = false;; again = true) {
                float squares = 0.0f;
                dot = 0.0f;
#pragma unroll
                for (int p = 0; p < PPL; ++p)
#pragma unroll
                    for (int e = 0; e < VE; ++e)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            squares = __builtin_fmaf(f[p][i][e], f[p][i][e], squares);
                            if constexpr (BACK) dot = __builtin_fmaf(w[p][i][e] * d[p][i][e], f[p][i][e], dot);
                        }
                squares = head_sum(squares, log);
                if constexpr (BACK) dot = head_sum(dot, log);
                mean = __builtin_fmaf(squares, scale, again ? __builtin_ldexpf(n.eps, -2 * down) : n.eps);
                const bool fits = mean >= (BACK ? SMALL_BACK : SMALL) && mean <= (BACK ? LARGE_BACK : LARGE);
                if (again || !__any(!fits)) break;
                // (lanes of heads that need none have down = 0, and get the same again)
                if (!fits) {
                    float top = 0.0f;
#pragma unroll
                    for (int p = 0; p < PPL; ++p)
#pragma unroll
                        for (int e = 0; e < VE; ++e) top = fmaxf(top, fmaxf(fabsf(f[p][0][e]), fabsf(f[p][1][e])));
                    const int e0 = exponent(head_max(top, log)), e1 = n.eps > 0.0f ? exponent(n.eps) / 2 : -127;
                    down = e0 > e1 ? e0 : e1;
#pragma unroll
                    for (int p = 0; p < PPL; ++p)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int e = 0; e < VE; ++e) f[p][i][e] = __builtin_ldexpf(f[p][i][e], -down);
                }
            }
            // (within one unit in the last place; of a head that is not there all is zero then)
            const float r = there ? __builtin_amdgcn_rsqf(mean) : 0.0f;
            if constexpr (BACK) dot = dot * r * scale;
            T* dst = (T*)head_at(!side, j.q_out, j.k_out, h);
            const bool stored = (side ? j.k_out.data : j.q_out.data) != nullptr;
            if constexpr (BACK) {
                auto add = [&](int v, float to) {
                    const int p = v / (2 * VE), i = v / VE % 2, e = v % VE;
                    return __builtin_fmaf(d[p][i][e], f[p][i][e] * r, to);
                };
                if (!side) {
#pragma unroll
                    for (int v = 0; v < VALUES; ++v) sum[v] = add(v, sum[v]);
                } else {
#pragma unroll
                    for (int v = 0; v < VALUES; v += 4) {
                        const f32x4 to = s_keys[v / 4][tid];
                        s_keys[v / 4][tid] = f32x4{add(v, to[0]), add(v + 1, to[1]), add(v + 2, to[2]), add(v + 3, to[3])};
                    }
                }
            }
#pragma unroll
            for (int p = 0; p < PPL; ++p) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        const float norm = f[p][i][e] * r;
                        if constexpr (!BACK) f[p][i][e] = norm * w[p][i][e];
                        else {
                            f[p][i][e] = r * __builtin_fmaf(-norm, dot, w[p][i][e] * d[p][i][e]);
                            if (down != 0) f[p][i][e] = __builtin_ldexpf(f[p][i][e], -down);
                        }
                    }
                if constexpr (!BACK) turn_by<VE, ADJACENT>(at[p], !CACHED || turns[p], f[p][0], f[p][1]);
                if (!there || !stored) continue;
                V y, z;
#pragma unroll
                for (int e = 0; e < VE; ++e) { narrow(f[p][0][e], y.e[e]); narrow(f[p][1][e], z.e[e]); }
                if (has_a[p]) store_once<CACHED>(y, dst + first[p]);
                if (has_b[p]) store_once<CACHED>(z, dst + second[p]);
            }
        };
        for (int base = 0; base < sh.steps;) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                if (base + u >= sh.steps) continue;
                take(u, base + u);
            }
            base += BATCH;
            if (base < sh.steps) fetch(base);
        }
    }
    if constexpr (BACK) {
        if (!n.sums) return;
        // this workgroup's row of sums: over the slots of a wavefront, pair by pair, then over its wavefronts
        __syncthreads();
        float* s_sum = reinterpret_cast<float*>(s_dyn);
#pragma unroll
        for (int side = 0; side < 2; ++side)
#pragma unroll
            for (int p = 0; p < PPL; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        const int at = (p * 2 + i) * VE + e;
                        float v = side ? s_keys[at / 4][tid][at % 4] : sum[at];
                        for (int k = log; k < 6; ++k) v += __shfl_xor(v, 1 << k);
                        const int d = (i ? second[p] : first[p]) + e;
                        const bool has = i ? has_b[p] : has_a[p];
                        if (slot == 0 && has) s_sum[(wave * 2 + side) * dim + d] = v;
                    }
        __syncthreads();
        for (int d = tid; d < 2 * dim; d += THREADS) {
            float v = 0.0f;
            for (int k = 0; k < WAVES; ++k) v += s_sum[k * 2 * dim + d];
            n.sums[(long)blockIdx.x * 2 * dim + d] = v;
        }
    }
}

// The workgroups' rows of sums, added up: 16 columns a workgroup, 64 threads a column, each of which takes every 64th row.
constexpr int COLUMNS = 16, TEAMS = 64;
__global__ __launch_bounds__(COLUMNS * TEAMS) void sums_kernel(const NormJob n, int rows)
{
    __shared__ double s_part[TEAMS][COLUMNS + 1];
    const int dim = n.r.dim, x = threadIdx.x % COLUMNS, col = blockIdx.x * COLUMNS + x, team = threadIdx.x / COLUMNS;
    float v[NORM_GROUPS / TEAMS];
#pragma unroll
    for (int i = 0; i < NORM_GROUPS / TEAMS; ++i) {
        const int row = team + TEAMS * i;
        v[i] = col < 2 * dim && row < rows ? n.sums[(long)row * 2 * dim + col] : 0.0f;
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < NORM_GROUPS / TEAMS; ++i) sum += v[i];
    s_part[team][x] = sum;
    for (int half = TEAMS / 2; half > 0; half /= 2) {
        __syncthreads();
        if (team < half) s_part[team][x] += s_part[team + half][x];
    }
    void* to = col < dim ? n.q_weight_grad : n.k_weight_grad;
    if (team != 0 || col >= 2 * dim || !to) return;
    const int d = col < dim ? col : col - dim;
    sum = s_part[0][x];
    if (n.weight_bf16) narrow((float)sum, ((uint16_t*)to)[d]);
    else ((float*)to)[d] = (float)sum;
}

template <bool BACK> hipError_t launch(const NormJob& n, hipStream_t st)
{
    const RotaryJob& j = n.r;
    const int ve = vector_values<6>(j.bf16, j.pairs, {&j.q, &j.q_out, &j.k, &j.k_out, &n.q_grad, &n.k_grad}), units = device_units();
    Shape sh;
    sh.pieces = (j.dim + 2 * ve - 1) / (2 * ve);
    sh.lanes_log = 0;
    while (1 << sh.lanes_log < sh.pieces && sh.lanes_log < 6) ++sh.lanes_log;
    // heads at a time: as many as leave the fewest lanes without one
    long least = LONG_MAX;
    for (int log = 0; log <= 6 - sh.lanes_log; ++log) {
        const int q = (j.q.heads + (1 << log) - 1) >> log, k = (j.k.heads + (1 << log) - 1) >> log;
        const long cost = (long)(q + k) << log;
        if (cost > least) continue;
        least = cost;
        sh.heads_log = log;
        sh.q_steps = q;
        sh.steps = q + k;
    }
    const int tokens = (64 >> sh.lanes_log) >> sh.heads_log;
    sh.stretches = (j.tokens + tokens - 1) / tokens;
    // backward as many workgroups as are at work at once, three a compute unit (19 200 tokens, 40 heads of 128 in bfloat16: 118 us, 129 with two); forward a
    // wavefront for every stretch (129 us, 136 - 143 with fewer)
    const long groups = (sh.stretches + WAVES - 1) / WAVES, at_once = 3L * units, most = BACK ? (at_once < NORM_GROUPS ? at_once : NORM_GROUPS) : 1L << 22;
    const dim3 grid((unsigned)(groups < most ? groups : most)), block(THREADS);
    size_t lds = (size_t)WAVES * tokens * j.pairs * sizeof(float2);
    if (BACK && lds < WAVES * 2 * j.dim * sizeof(float)) lds = WAVES * 2 * j.dim * sizeof(float);
    // Around the caches where a load or store of a wavefront has whole lines, or nearly so: first and second values of pairs apart, each of 128, 192 or more
    // bytes.  Where two of them share the lines, the caches bring these together.  (19 200 tokens, 40 heads in bfloat16, around and through the caches: halves of
    // 128 values 68 and 76 us, 64: 46 and 43, 96: 73 and 62, adjacent pairs of 128: 112 and 78, gradients 146 and 131; 9 600 tokens in float32, halves of 64: 36 and
    // 42, 80: 57 and 54, 96: 60 and 62, adjacent pairs of 128: 131 and 84.)
    const int half = j.pairs * (j.bf16 ? 2 : 4);
    const bool around = !j.adjacent && 2 * j.pairs == j.dim && ve * (j.bf16 ? 2 : 4) == 16 && (half == 128 || half >= 192);
#define CB_NORM(type, v, p, adjacent, cached) hipLaunchKernelGGL((norm_kernel<type, v, p, adjacent, cached, BACK>), grid, block, lds, st, n, sh)
#define CB_NORMS(type, v) do { if (j.adjacent) CB_NORM(type, v, 1, true, true); else CB_NORM(type, v, 1, false, true); } while (0)
    if (j.bf16) {
        if (around) CB_NORM(uint16_t, 8, 1, false, false);
        else if (ve == 8) CB_NORMS(uint16_t, 8);
        else if (ve == 4) CB_NORMS(uint16_t, 4);
        else if (ve == 2) CB_NORMS(uint16_t, 2);
        else CB_NORM(uint16_t, 1, 2, false, true);
    } else {
        if (around) CB_NORM(float, 4, 1, false, false);
        else if (ve == 4) CB_NORMS(float, 4);
        else if (ve == 2) CB_NORMS(float, 2);
        else CB_NORM(float, 1, 2, false, true);
    }
#undef CB_NORMS
#undef CB_NORM
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !BACK || !n.sums) return e;
    hipLaunchKernelGGL(sums_kernel, dim3((2 * j.dim + COLUMNS - 1) / COLUMNS), dim3(COLUMNS * TEAMS), 0, st, n, (int)grid.x);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rotate(const NormJob& n, hipStream_t st) { return n.r.tokens ? launch<false>(n, st) : hipSuccess; }

// (no tokens: the weights' gradients are zero, which the sums over no rows are)
hipError_t launch_norm_rotate_back(const NormJob& n, hipStream_t st)
{
    if (n.r.tokens) return launch<true>(n, st);
    if (!n.sums) return hipSuccess;
    hipLaunchKernelGGL(sums_kernel, dim3((2 * n.r.dim + COLUMNS - 1) / COLUMNS), dim3(COLUMNS * TEAMS), 0, st, n, 0);
    return hipGetLastError();
}

}  // namespace cb
