// Appending to a cache in 8 bits: e4m3 values with a float32 scale for every 16 tokens ("block") of a page and key head, of keys and of values.
//
// The scale is the smallest power of two, 2^-64 at least, of which 448 times (e4m3's largest) reaches every finite value of the block, and no smaller
// than that of the tokens that are there already; where it grows, these are rounded again, which is exact for all that do not become subnormal.
// Powers of two keep a value's relative error at half a step of e4m3 whatever its block holds, and let every product and quotient with a scale be exact.
// (A scale that a caller has written may be any number: the values are divided by it then.)
//
// A block and a head belong to one wavefront: it reads the new tokens' rows, turns keys, takes the maximum across its lanes from registers,
// and writes 16 rows of a page that lie one behind the other.  Memory bounds it: 2 or 4 bytes read and 1 written a value (35 000 tokens of 8 heads of 128 in
// bfloat16: 40 us, 5.4 TB/s).  One token for each of 16 sequences takes 3.8 us, trips to memory one behind the other: start, page, rows and the scale that is there.
// A workgroup has one block of tokens, whose angles it makes once, and some or all of its heads.  Which block of which sequence the device finds
// itself: sequence s has the numbers from offsets[s] / 16 + 2 s on, which leaves room for one begun block in front and one behind.
#include "cb_rows.h"

namespace cb {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64, BLOCK = 16;
constexpr float MOST = 448.0f;

// The smallest power of two, in -64 .. 120, of which 448 = 1.75 * 2^8 times is `top` at least.
__device__ __forceinline__ float scale_for(float top)
{
    const uint32_t b = __float_as_uint(top);
    int e = (int)(b >> 23) - 126 - ((b & 0x7FFFFFu) <= 0x600000u ? 9 : 8);
    e = e < -64 ? -64 : (e > 120 ? 120 : e);
    return __uint_as_float((uint32_t)(127 + e) << 23);
}

template <int VE> struct Codes { uint8_t e[VE]; };
// VE values, none above the largest that 8 bits hold, as codes: to the nearest, ties to even; what is not a number stays so
template <int VE> __device__ __forceinline__ void encode(const float (&f)[VE], uint8_t* to)
{
    if constexpr (VE == 1) *to = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[0], 0.0f, 0, false);
    else if constexpr (VE == 2) *reinterpret_cast<uint16_t*>(to) = (uint16_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    else {
        uint32_t w[VE / 4];
#pragma unroll
        for (int i = 0; i < VE / 4; ++i) {
            const int low = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
            w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], low, true);
        }
        if constexpr (VE == 4) *reinterpret_cast<uint32_t*>(to) = w[0];
        else *reinterpret_cast<uint64_t*>(to) = (uint64_t)w[1] << 32 | w[0];
    }
}
template <int VE> __device__ __forceinline__ void decode(const uint8_t* from, float (&f)[VE])
{
#pragma unroll
    for (int i = 0; i < VE; ++i) f[i] = __builtin_amdgcn_cvt_f32_fp8((int)from[i], 0);
}

template <typename T, int VE, int DP>
__global__ __launch_bounds__(THREADS) void append_bytes_kernel(const RotaryJob j, const Cache c, int pieces, int lengths)
{
    typedef Vec<T, VE> V;
    typedef typename Word<sizeof(V)>::type W;
    constexpr int ITEMS = DP / (8 * VE);         // of a lane: (token, piece of its row), two vectors each
    extern __shared__ float2 cs[];               // BLOCK x pairs
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), np = j.pairs, turned = np / VE;

    // the sequence and its rows
    int seq = blockIdx.x, block = 0;
    long row0 = blockIdx.x, rows = 1;
    bool there = true;
    if (j.offsets) {
        auto at = [&](int s) { const int o = j.offsets[s]; return o < 0 ? 0L : (o > j.tokens ? j.tokens : (long)o); };
        int lo = 0, hi = c.seqs - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (at(mid) / BLOCK + 2L * mid <= (long)blockIdx.x) lo = mid; else hi = mid - 1;
        }
        seq = lo;
        row0 = at(seq);
        rows = at(seq + 1) - row0;
        const long first = row0 / BLOCK + 2L * seq;
        there = (long)blockIdx.x >= first;
        block = (int)((long)blockIdx.x - first);
    }
    const int start = clamp_length(j.start[seq], c.capacity);
    const long slot0 = ((long)start / BLOCK + block) * BLOCK;          // of the block's first token
    // new tokens are those from `from` to `to` - 1 of the block; in front of them lie tokens that were there
    const int from = start > slot0 ? (int)(start - slot0) : 0;
    const long left = start + rows - slot0;
    const int to = left < BLOCK ? (int)left : BLOCK;
    there = there && rows > 0 && from < to && slot0 < c.capacity;
    const long token0 = row0 + (slot0 - start);                        // row of the block's first token, if it is a new one
    int page = -1;
    if (there) page = c.table[(long)seq * c.max_pages + (slot0 >> c.page_shift)];
    if (there && np) {
        for (int i = tid; i < BLOCK * np; i += THREADS) {
            const int t = i / np;
            if (t >= from && t < to) cs[i] = angle_of(j, token0 + t, i - t * np);
        }
    }
    __syncthreads();
    if (lengths == LENGTHS_FIRST) {
        if (blockIdx.x == 0 && blockIdx.y == 0) set_lengths(j, c, tid, THREADS);
    } else if (lengths == LENGTHS_LAST) {
        // start is lengths itself: every workgroup has read it (above) before the last one writes it
        if (tid == 0) {
            int* counter = reinterpret_cast<int*>(c.scratch);
            last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)(gridDim.x * gridDim.y) - 1;
            if (last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (last) set_lengths(j, c, tid, THREADS);
    }
    if (!there) return;
    if (blockIdx.y == 0 && (c.weight || c.time))
        for (int i = tid; i < BLOCK * c.heads; i += THREADS) {
            const int h = i / BLOCK, t = i - h * BLOCK;
            if (t < from || t >= to) continue;
            const long at = ((long)seq * c.heads + h) * c.capacity + slot0 + t;
            if (c.weight) c.weight[at] = 0.0f;
            if (c.time) c.time[at] = j.positions ? j.positions[(token0 + t) * j.pos_axes] : (int)(slot0 + t);
        }
    if ((unsigned)page >= (unsigned)c.n_pages) return;

    // where a lane's items lie: token and piece of its row
    int token[ITEMS], piece[ITEMS];
    bool is_new[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        token[i] = (lane + 64 * i) / pieces;
        piece[i] = lane + 64 * i - token[i] * pieces;
        is_new[i] = token[i] >= from && token[i] < to;
    }
    // rows of which nothing turns are taken by halves, where these are whole vectors: a load or store of the wavefront has whole lines then, not every
    // other 16 bytes (45.7 -> 43.8 us)
    const int half = c.dim % (2 * VE) == 0 ? c.dim / 2 : 0;
    auto first_of = [&](bool key, int i) {
        const bool turns = key && piece[i] < turned;
        return (turns && !j.adjacent) || (!(key && np) && half) ? VE * piece[i] : 2 * VE * piece[i];
    };
    auto second_of = [&](bool key, int i) {
        const bool turns = key && piece[i] < turned;
        return !(key && np) && half ? half + VE * piece[i] : (turns && !j.adjacent ? np + VE * piece[i] : 2 * VE * piece[i] + VE);
    };
    W raw[ITEMS][2];
    auto fetch = [&](int unit) {
        const bool key = unit < c.heads;
        const T* src = (const T*)(key ? j.k.data : j.v.data) + (long)(key ? unit : unit - c.heads) * (key ? j.k.head : j.v.head);
        const long stride = key ? j.k.token : j.v.token;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const T* row = src + (token0 + token[i]) * stride;
            auto get = [](bool there, const T* from) {
                W v = W{};
                if (there) v = *reinterpret_cast<const W*>(from);
                return v;
            };
            raw[i][0] = get(is_new[i], row + first_of(key, i));
            raw[i][1] = get(is_new[i] && second_of(key, i) < c.dim, row + second_of(key, i));
        }
    };
    for (int unit = blockIdx.y * WAVES + wave; unit < 2 * c.heads; unit += gridDim.y * WAVES) {
        const bool key = unit < c.heads;
        const int h = key ? unit : unit - c.heads;
        const long head = (long)page * c.heads + h;
        uint8_t* dst = (uint8_t*)(key ? c.k : c.v) + ((head << c.page_shift) + (slot0 & ((1 << c.page_shift) - 1))) * c.dim;
        float* scale_at = (key ? c.k_scale : c.v_scale) + (head << (c.page_shift - 4)) + ((slot0 & ((1 << c.page_shift) - 1)) >> 4);
        const float old = from > 0 ? *scale_at : 0.0f;
        fetch(unit);
        float f[ITEMS][2][VE];
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const V a = __builtin_bit_cast(V, raw[i][0]), b = __builtin_bit_cast(V, raw[i][1]);
#pragma unroll
            for (int e = 0; e < VE; ++e) { f[i][0][e] = widen(a.e[e]); f[i][1][e] = widen(b.e[e]); }
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (key && piece[i] < turned && is_new[i]) turn<VE>(cs + token[i] * np + piece[i] * VE, j.adjacent, f[i][0], f[i][1]);
#pragma unroll
            for (int e = 0; e < VE; ++e) top = fmaxf(top, fmaxf(fabsf(f[i][0][e]), fabsf(f[i][1][e])));      // (what is not a number is passed over)
        }
        top = wave_max(top);
        const bool infinite = top == __builtin_inff();
        if (infinite) {
            top = 0.0f;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int e = 0; e < VE; ++e)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float size = fabsf(f[i][x][e]);
                        top = fmaxf(top, size < __builtin_inff() ? size : 0.0f);
                    }
            top = wave_max(top);
        }
        const float need = scale_for(top), now = from > 0 ? fmaxf(need, old) : need;
        const uint32_t bits = __float_as_uint(now);
        const bool exact = (bits & 0x7FFFFFu) == 0 && bits >= 0x00800000u && bits <= 0x7E000000u;      // 2^-126 .. 2^125: so is its inverse
        const float inverse = exact ? __uint_as_float(0x7F000000u - bits) : 0.0f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int first = first_of(key, i), second = second_of(key, i);
            uint8_t* row = dst + (long)token[i] * c.dim;
            if (token[i] < from && now != old) {
                const float ratio = old / now;
                decode<VE>(row + first, f[i][0]);
                if (second < c.dim) decode<VE>(row + second, f[i][1]);
#pragma unroll
                for (int e = 0; e < VE; ++e) { f[i][0][e] *= ratio; f[i][1][e] *= ratio; }
            } else if (is_new[i]) {
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    f[i][0][e] = exact ? f[i][0][e] * inverse : f[i][0][e] / now;
                    f[i][1][e] = exact ? f[i][1][e] * inverse : f[i][1][e] / now;
                }
                if (infinite)
#pragma unroll
                    for (int e = 0; e < VE; ++e)
#pragma unroll
                        for (int x = 0; x < 2; ++x) f[i][x][e] = f[i][x][e] == f[i][x][e] ? __builtin_amdgcn_fmed3f(f[i][x][e], -MOST, MOST) : f[i][x][e];
            } else continue;
            encode<VE>(f[i][0], row + first);
            if (second < c.dim) encode<VE>(f[i][1], row + second);
        }
        if (lane == 0) *scale_at = now;
    }
}

template <typename T, int VE> void launch_as(const RotaryJob& j, const Cache& c, dim3 grid, int pieces, int lengths, hipStream_t st)
{
    const size_t lds = (size_t)BLOCK * j.pairs * sizeof(float2);
#define CB_APPEND(d) hipLaunchKernelGGL((append_bytes_kernel<T, VE, d>), grid, dim3(THREADS), lds, st, j, c, pieces, lengths)
    if (c.dim <= 64) CB_APPEND(64);
    else if (c.dim <= 128) CB_APPEND(128);
    else CB_APPEND(256);
#undef CB_APPEND
}

}  // namespace

hipError_t launch_append_bytes(const RotaryJob& j, const Cache& c, int* lengths, hipStream_t st)
{
    const int ve = vector_values<2>(j.bf16, j.pairs, {&j.k, &j.v}), pieces = (c.dim + 2 * ve - 1) / (2 * ve);
    const long blocks = j.offsets ? j.tokens / BLOCK + 2L * c.seqs : c.seqs;
    // a wavefront a head where there are few blocks, two heads where there are many (42 us with four or eight)
    const int units = 2 * c.heads, most = (units + WAVES - 1) / WAVES;
    int split = most;
    while (split > 1 && blocks * (split / 2) >= 4L * device_units() && most / (split / 2) <= 2) split /= 2;
    const dim3 grid((unsigned)blocks, (unsigned)split);
    if (*lengths == LENGTHS_LAST && blocks * split > 64) *lengths = LENGTHS_LATER;
    if (j.bf16) {
        if (ve == 8) launch_as<uint16_t, 8>(j, c, grid, pieces, *lengths, st);
        else if (ve == 4) launch_as<uint16_t, 4>(j, c, grid, pieces, *lengths, st);
        else if (ve == 2) launch_as<uint16_t, 2>(j, c, grid, pieces, *lengths, st);
        else launch_as<uint16_t, 1>(j, c, grid, pieces, *lengths, st);
    } else {
        if (ve == 4) launch_as<float, 4>(j, c, grid, pieces, *lengths, st);
        else if (ve == 2) launch_as<float, 2>(j, c, grid, pieces, *lengths, st);
        else launch_as<float, 1>(j, c, grid, pieces, *lengths, st);
    }
    return hipGetLastError();
}

}  // namespace cb
