// Norms of heads with their rotation in the same pass, and the gradients of both.
//
// A head x of D values: n = x r, r = (mean x^2 + eps)^-1/2, out = R(n w), where w has a weight for every value and R turns pairs by the token's
// position (cb_rotary.hip).  Backward, with g = R^-1(gradient of out): the gradient of x is r (w g - n mean(w g n)), that of w the sum over tokens and
// heads of g n.  Since mean(w g n) = r mean(w g x), both sums over a head are made in one go.
//
// Heads are independent and read once, so memory bounds it: 2 values' bytes forward, 3 backward.  A head lies in the registers of 1 - 64 lanes (two
// vectors of 16 bytes a lane, as pairs need them), its sums take a few steps across them, and a workgroup makes its tokens' angles once for all heads.
// A gradient of the weights is summed in registers by persistent workgroups, each of which leaves one row of sums; a second launch adds these
// up in order, so that results do not vary.
#include "cb_rows.h"

namespace cb {

namespace {

constexpr int THREADS = 256;
constexpr int MAX_ANGLES = 512;                  // of a workgroup
constexpr int MAX_TOKENS = 16;
constexpr int MAX_DIM = 256;
// Mean squares in float32 are exact enough, and their root's inverse is a normal number, between these; what is beyond is computed in float64.
constexpr float SMALL = 0x1p-100f, LARGE = 0x1p100f;

struct Shape {
    int tokens;                    // of a workgroup at a time
    int pieces, lanes_log;         // two vectors a piece; lanes of a head
    long steps;                    // stretches of `tokens`
};

__device__ __forceinline__ float weight_of(const void* w, int bf16, int i)
{
    return bf16 ? widen(((const uint16_t*)w)[i]) : ((const float*)w)[i];
}

// The sum over the 2^log lanes of a head, the same in each: partners' sums are added in both lanes of a pair.
__device__ __forceinline__ float head_sum(float v, int log)
{
    auto add = [](float a, int b) { return a + __uint_as_float((uint32_t)b); };
    if (log > 0) v = add(v, __builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0xB1, 0xf, 0xf, true));      // quad_perm 1 0 3 2
    if (log > 1) v = add(v, __builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x4E, 0xf, 0xf, true));      // quad_perm 2 3 0 1
    if (log > 2) v = add(v, __builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x141, 0xf, 0xf, true));     // row_half_mirror
    if (log > 3) v = add(v, __builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x140, 0xf, 0xf, true));     // row_mirror
    if (log > 4) v += __shfl_xor(v, 16);
    if (log > 5) v += __shfl_xor(v, 32);
    return v;
}
__device__ __forceinline__ double head_sum(double v, int log)
{
    for (int i = 0; i < log; ++i) v += __shfl_xor(v, 1 << i);
    return v;
}

// PPL: pieces of a head that a lane has (more than one where single values are taken of heads above 128).
template <typename T, int VE, int PPL, bool BACK>
__global__ __launch_bounds__(THREADS) void norm_kernel(const NormJob n, const Shape sh)
{
    typedef Vec<T, VE> V;
    // heads of a lane's group that are on their way at once
    constexpr int BATCH = BACK ? 2 : 3;
    __shared__ float2 cs[MAX_ANGLES];
    __shared__ __align__(16) float s_w[2][MAX_DIM];
    extern __shared__ float s_sum[];             // BACK: 2 * VE * PPL values of every thread
    const RotaryJob& j = n.r;
    const int tid = threadIdx.x, np = j.pairs, dim = j.dim, hq = j.q.heads, heads = hq + j.k.heads;
    const int lanes_log = sh.lanes_log, group = tid >> lanes_log, groups = THREADS >> lanes_log, sub = tid & ((1 << lanes_log) - 1);
    const int turned = np / VE;
    const float scale = 1.0f / (float)dim;
    for (int i = tid; i < 2 * dim; i += THREADS) {
        const void* w = i < dim ? n.q_weight : n.k_weight;
        const int d = i < dim ? i : i - dim;
        s_w[i < dim ? 0 : 1][d] = w ? weight_of(w, n.weight_bf16, d) : 0.0f;
    }
    // where a lane's pieces lie in a head, the same of every head
    int first[PPL], second[PPL];
    bool turns[PPL], has_a[PPL], has_b[PPL];
#pragma unroll
    for (int p = 0; p < PPL; ++p) {
        const int piece = sub + (p << lanes_log);
        turns[p] = piece < turned;
        first[p] = turns[p] && !j.adjacent ? VE * piece : 2 * VE * piece;
        second[p] = turns[p] && !j.adjacent ? np + VE * piece : 2 * VE * piece + VE;
        has_a[p] = piece < sh.pieces;
        has_b[p] = has_a[p] && second[p] < dim;
    }
    float sum_q[PPL][2][VE] = {}, sum_k[PPL][2][VE] = {};        // BACK: of g n, of all heads that were here

    for (long step = blockIdx.x; step < sh.steps; step += gridDim.x) {
        const long tok0 = step * sh.tokens;
        const int here = (int)(j.tokens - tok0 < sh.tokens ? j.tokens - tok0 : sh.tokens), rows = here * heads;
        V x[BATCH][PPL][2], g[BATCH][PPL][2];
        auto fetch = [&](int base) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int row = base + u * groups, t = row / heads, h = row - t * heads;
                const bool q = h < hq, there = row < rows;
                const Heads& from = q ? j.q : j.k;
                const T* src = (const T*)from.data + (tok0 + t) * from.token + (long)(q ? h : h - hq) * from.head;
                const Heads& grad = q ? n.q_grad : n.k_grad;
                const T* gsrc = BACK ? (const T*)grad.data + (tok0 + t) * grad.token + (long)(q ? h : h - hq) * grad.head : nullptr;
#pragma unroll
                for (int p = 0; p < PPL; ++p) {
                    x[u][p][0] = x[u][p][1] = V{};
                    if (there && has_a[p]) x[u][p][0] = load_once<false, V>(src + first[p]);
                    if (there && has_b[p]) x[u][p][1] = load_once<false, V>(src + second[p]);
                    if constexpr (BACK) {
                        g[u][p][0] = g[u][p][1] = V{};
                        if (there && has_a[p]) g[u][p][0] = load_once<false, V>(gsrc + first[p]);
                        if (there && has_b[p]) g[u][p][1] = load_once<false, V>(gsrc + second[p]);
                    }
                }
            }
        };
        fetch(group);
        __syncthreads();                         // the last stretch's angles have been used
        for (int i = tid; i < here * np; i += THREADS) {
            const int t = i / np;
            cs[i] = angle_of(j, tok0 + t, i - t * np);
        }
        __syncthreads();
        for (int base = group; base - group < rows;) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int row = base + u * groups, t = row / heads, h = row - t * heads;
                const bool q = h < hq, there = row < rows;
                if (base - group + u * groups >= rows) break;        // (the same for all: lanes of a head add up together)
                const float* w = s_w[q ? 0 : 1];
                const float2* at = cs + (there ? t : 0) * np;
                float f[PPL][2][VE], d[PPL][2][VE];                  // the head; BACK: w times its gradient, turned back
                float squares = 0.0f, dot = 0.0f;
#pragma unroll
                for (int p = 0; p < PPL; ++p) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        f[p][0][e] = widen(x[u][p][0].e[e]);
                        f[p][1][e] = widen(x[u][p][1].e[e]);
                        if constexpr (BACK) {
                            d[p][0][e] = widen(g[u][p][0].e[e]);
                            d[p][1][e] = widen(g[u][p][1].e[e]);
                        }
                        squares += f[p][0][e] * f[p][0][e];
                        squares += f[p][1][e] * f[p][1][e];
                    }
                    if constexpr (BACK) {
                        if (turns[p]) turn<VE>(at + (sub + (p << lanes_log)) * VE, j.adjacent, d[p][0], d[p][1]);
#pragma unroll
                        for (int e = 0; e < VE; ++e) {
                            if (has_a[p]) dot += w[first[p] + e] * d[p][0][e] * f[p][0][e];
                            if (has_b[p]) dot += w[second[p] + e] * d[p][1][e] * f[p][1][e];
                        }
                    }
                }
                squares = head_sum(squares, lanes_log);
                const float mean = squares * scale + n.eps;
                float r = 0.0f;
                double r64 = 0.0, dot64 = 0.0;
                const bool far = !(mean >= SMALL && mean <= LARGE);
                if (!far) {
                    r = 1.0f / sqrtf(mean);
                    if constexpr (BACK) dot = head_sum(dot, lanes_log) * r * scale;
                } else {
                    double sum = 0.0;
#pragma unroll
                    for (int p = 0; p < PPL; ++p)
#pragma unroll
                        for (int e = 0; e < VE; ++e) {
                            sum += (double)f[p][0][e] * f[p][0][e] + (double)f[p][1][e] * f[p][1][e];
                            if constexpr (BACK) {
                                if (has_a[p]) dot64 += (double)w[first[p] + e] * d[p][0][e] * f[p][0][e];
                                if (has_b[p]) dot64 += (double)w[second[p] + e] * d[p][1][e] * f[p][1][e];
                            }
                        }
                    r64 = 1.0 / sqrt(head_sum(sum, lanes_log) / dim + (double)n.eps);
                    dot64 = head_sum(dot64, lanes_log) * r64 / dim;
                }
                const Heads& to = q ? j.q_out : j.k_out;
                T* dst = (T*)to.data + (tok0 + t) * to.token + (long)(q ? h : h - hq) * to.head;
#pragma unroll
                for (int p = 0; p < PPL; ++p) {
#pragma unroll
                    for (int e = 0; e < VE; ++e)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int at = (i ? second[p] : first[p]) + e;
                            const float wi = (i ? has_b[p] : has_a[p]) ? w[at] : 0.0f;
                            if constexpr (!BACK) f[p][i][e] = far ? (float)((double)f[p][i][e] * r64 * wi) : f[p][i][e] * r * wi;
                            else {
                                const float norm = far ? (float)((double)f[p][i][e] * r64) : f[p][i][e] * r, part = d[p][i][e] * norm;
                                if (q) sum_q[p][i][e] += there ? part : 0.0f;
                                else sum_k[p][i][e] += there ? part : 0.0f;
                                f[p][i][e] = far ? (float)(r64 * ((double)wi * d[p][i][e] - norm * dot64)) : r * (wi * d[p][i][e] - norm * dot);
                            }
                        }
                    if (!BACK && turns[p]) turn<VE>(at + (sub + (p << lanes_log)) * VE, j.adjacent, f[p][0], f[p][1]);
                    if (!there || !to.data) continue;
                    V y, z;
#pragma unroll
                    for (int e = 0; e < VE; ++e) { narrow(f[p][0][e], y.e[e]); narrow(f[p][1][e], z.e[e]); }
                    if (has_a[p]) store_once<false>(y, dst + first[p]);
                    if (has_b[p]) store_once<false>(z, dst + second[p]);
                }
            }
            base += BATCH * groups;
            if (base - group < rows) fetch(base);
        }
    }
    if constexpr (BACK) {
        if (!n.sums) return;
        // this workgroup's row of sums: over its groups of lanes, in order
        constexpr int OWN = 2 * VE * PPL;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            __syncthreads();
#pragma unroll
            for (int p = 0; p < PPL; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < VE; ++e) s_sum[((p * 2 + i) * VE + e) * THREADS + tid] = side ? sum_k[p][i][e] : sum_q[p][i][e];
            __syncthreads();
            for (int o = tid; o < OWN << lanes_log; o += THREADS) {
                const int slot = o >> lanes_log, lane = o & ((1 << lanes_log) - 1), e = slot % VE, i = slot / VE % 2, piece = lane + ((slot / (2 * VE)) << lanes_log);
                if (piece >= sh.pieces) continue;
                const bool t = piece < turned && !j.adjacent;
                const int d = (i == 0 ? (t ? VE * piece : 2 * VE * piece) : (t ? np + VE * piece : 2 * VE * piece + VE)) + e;
                if (d >= dim) continue;
                float sum = 0.0f;
                for (int y = 0; y < groups; ++y) sum += s_sum[slot * THREADS + (y << lanes_log) + lane];
                n.sums[((long)blockIdx.x * 2 + side) * dim + d] = sum;
            }
        }
    }
}

// The workgroups' rows of sums, added up: 16 columns a workgroup, 16 threads a column, each of which takes every 16th row.
__global__ __launch_bounds__(256) void sums_kernel(const NormJob n, int rows)
{
    __shared__ double s_part[16][16];
    const int dim = n.r.dim, col = blockIdx.x * 16 + (threadIdx.x & 15), team = threadIdx.x >> 4;
    double sum = 0.0;
    if (col < 2 * dim)
        for (int i = team; i < rows; i += 16) sum += n.sums[(long)i * 2 * dim + col];
    s_part[team][threadIdx.x & 15] = sum;
    __syncthreads();
    if (team != 0 || col >= 2 * dim) return;
    for (int i = 1; i < 16; ++i) sum += s_part[i][threadIdx.x & 15];
    void* to = col < dim ? n.q_weight_grad : n.k_weight_grad;
    const int d = col < dim ? col : col - dim;
    if (!to) return;
    if (n.weight_bf16) narrow((float)sum, ((uint16_t*)to)[d]);
    else ((float*)to)[d] = (float)sum;
}

template <bool BACK> hipError_t launch(const NormJob& n, hipStream_t st)
{
    const RotaryJob& j = n.r;
    const int ve = vector_values<6>(j.bf16, j.pairs, {&j.q, &j.q_out, &j.k, &j.k_out, &n.q_grad, &n.k_grad});
    Shape sh;
    sh.pieces = (j.dim + 2 * ve - 1) / (2 * ve);
    sh.lanes_log = 0;
    while (1 << sh.lanes_log < sh.pieces && sh.lanes_log < 6) ++sh.lanes_log;
    const int heads = j.q.heads + j.k.heads, at_once = (BACK ? 2 : 3) * (THREADS >> sh.lanes_log), angles = MAX_ANGLES / j.pairs, units = device_units();
    int tt = at_once / heads;
    tt = tt < angles ? tt : angles;
    tt = tt < 1 ? 1 : (tt > MAX_TOKENS ? MAX_TOKENS : tt);
    while (tt > 1 && j.tokens / tt < 4L * units) tt /= 2;
    sh.tokens = tt;
    sh.steps = (j.tokens + tt - 1) / tt;
    const long most = BACK ? NORM_GROUPS : 1L << 22;
    const dim3 grid((unsigned)(sh.steps < most ? sh.steps : most)), block(THREADS);
#define CB_NORM(type, v, p) hipLaunchKernelGGL((norm_kernel<type, v, p, BACK>), grid, block, BACK ? 2 * v * p * THREADS * sizeof(float) : 0, st, n, sh)
    if (j.bf16) {
        if (ve == 8) CB_NORM(uint16_t, 8, 1);
        else if (ve == 4) CB_NORM(uint16_t, 4, 1);
        else if (ve == 2) CB_NORM(uint16_t, 2, 1);
        else CB_NORM(uint16_t, 1, 2);
    } else {
        if (ve == 4) CB_NORM(float, 4, 1);
        else if (ve == 2) CB_NORM(float, 2, 1);
        else CB_NORM(float, 1, 2);
    }
#undef CB_NORM
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !BACK || !n.sums) return e;
    hipLaunchKernelGGL(sums_kernel, dim3((2 * j.dim + 15) / 16), dim3(256), 0, st, n, (int)grid.x);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rotate(const NormJob& n, hipStream_t st) { return n.r.tokens ? launch<false>(n, st) : hipSuccess; }

// (no tokens: the weights' gradients are zero, which the sums over no rows are)
hipError_t launch_norm_rotate_back(const NormJob& n, hipStream_t st)
{
    if (n.r.tokens) return launch<true>(n, st);
    if (!n.sums) return hipSuccess;
    hipLaunchKernelGGL(sums_kernel, dim3((2 * n.r.dim + 15) / 16), dim3(256), 0, st, n, 0);
    return hipGetLastError();
}

}  // namespace cb
