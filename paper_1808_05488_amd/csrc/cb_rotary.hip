// Rotary positions with several axes, and the append to a paged cache that rotates keys (and queries) on its way.
//
// Pair p of a head, values x and y, turns by position[axis of p] * turns[p] turns: (x cos - y sin, x sin + y cos).  The angle belongs
// to the token, not to the head, so a workgroup takes a few tokens, computes each of their angles once into LDS, and
// then streams all heads of those tokens past them.  A value is read once and written once; memory bounds it: 38 400 tokens x 40 heads of 128
// in bfloat16 130 us (6.1 TB/s, reads and writes; a large copy reaches 5.4, around the caches 6.4), appending 35 000 tokens of 48 heads 172 us (5.0).  The first batch of values
// is on its way while the angles are made, and a workgroup ends with one batch: 137 us with four times the tokens.  One token for
// each of 16 sequences takes 5.6 us, the trips to memory for sequence, page, position and values one after the other.  (Appends to slots that are given;
// behind the tokens that are there, lengths change last: 0.7 us more for the 16 tokens, 2 for 6 126 tokens with a launch of its own.)
#include "cb_tokens.h"

namespace cb {

namespace {

constexpr int THREADS = 256;
constexpr int BATCH = 3;                         // items of a thread at a time
constexpr int MAX_TOKENS = 8;                    // of a workgroup
constexpr int MAX_ANGLES = 256;                  // of a workgroup

template <typename T, int VE> struct alignas(sizeof(T) * VE) Vec { T e[VE]; };

template <int BYTES> struct Word;
template <> struct Word<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <> struct Word<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<2> { typedef uint16_t type; };
// Values of a rotation pass through once: around the caches (38 400 x 40 heads of 128: 147 -> 137 us).  Those of an append
// end in rows of many pages, and are better gathered in the caches on their way (35 000 tokens, 48 heads: 176 us, 204 around them).
template <bool CACHED, typename V> __device__ __forceinline__ V load_once(const void* p)
{
    typedef typename Word<sizeof(V)>::type W;
    return CACHED ? *reinterpret_cast<const V*>(p) : __builtin_bit_cast(V, __builtin_nontemporal_load(reinterpret_cast<const W*>(p)));
}
template <bool CACHED, typename V> __device__ __forceinline__ void store_once(const V& v, void* p)
{
    typedef typename Word<sizeof(V)>::type W;
    if (CACHED) *reinterpret_cast<V*>(p) = v;
    else __builtin_nontemporal_store(__builtin_bit_cast(W, v), reinterpret_cast<W*>(p));
}

// Where a token goes in the cache.
struct Place {
    long row;      // value offset of head 0's row in the pages, -1: nowhere
    long slot;     // offset of head 0's weight and time, -1: nowhere
    int time;
    int ignored;   // a row behind the last sequence's
};

__device__ void find_place(const RotaryJob& j, const Cache& c, long tok, Place* place)
{
    int seq = (int)tok;
    long first = tok;
    place->row = place->slot = -1;
    place->ignored = 0;
    if (j.offsets) {
        // the last sequence whose rows begin at or before tok (empty ones begin there too)
        int lo = 0, hi = c.seqs;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (j.offsets[mid] <= tok) lo = mid; else hi = mid - 1;
        }
        seq = lo;
        first = j.offsets[seq < c.seqs ? seq : 0];
        if (seq >= c.seqs || first > tok) { place->ignored = 1; return; }
    }
    const long slot = (long)clamp_length(j.start[seq], c.capacity) + (tok - first);
    place->time = j.positions ? j.positions[tok * j.pos_axes] : (int)slot;
    if (slot >= c.capacity) return;
    const int page = c.table[(long)seq * c.max_pages + (slot >> c.page_shift)];
    place->slot = (long)seq * c.heads * c.capacity + slot;
    if ((unsigned)page >= (unsigned)c.n_pages) return;
    place->row = ((((long)page * c.heads) << c.page_shift) + (slot & ((1 << c.page_shift) - 1))) * c.dim;
}

// lengths after the call: start + rows, as far as there are such rows and room
__device__ void set_lengths(const RotaryJob& j, const Cache& c, int first, int step)
{
    for (int s = first; s < c.seqs; s += step) {
        long rows = 1;
        if (j.offsets) {
            const long a = j.offsets[s], b = j.offsets[s + 1] < j.tokens ? j.offsets[s + 1] : j.tokens;
            rows = b > a ? b - a : 0;
        }
        const long n = clamp_length(j.start[s], c.capacity) + rows;
        c.lengths[s] = n > c.capacity ? c.capacity : (int)n;
    }
}

__global__ __launch_bounds__(THREADS) void lengths_kernel(const RotaryJob j, const Cache c)
{
    set_lengths(j, c, blockIdx.x * THREADS + threadIdx.x, gridDim.x * THREADS);
}

enum { LENGTHS_LATER = 0, LENGTHS_FIRST = 1 /* first workgroup */, LENGTHS_LAST = 2 /* whoever has read start last */ };

// A workgroup's items are (token, head, piece): two vectors of VE values each.  Of the n pairs of a head, piece p < n / VE turns
// pairs p * VE .. p * VE + VE - 1; the pieces behind copy what lies behind the pairs, two vectors at a time.  So every
// head has `pieces` = ceil(dim / (2 * VE)) of them, turned or not.
template <typename T, int VE, bool PAGED>
__global__ __launch_bounds__(THREADS) void rotary_kernel(const RotaryJob j, const Cache c, int tt, int pieces, int lengths)
{
    typedef Vec<T, VE> V;
    __shared__ float2 cs[MAX_ANGLES];
    __shared__ Place place[MAX_TOKENS];
    __shared__ int last;
    const int tid = threadIdx.x, n = j.pairs;
    const long tok0 = (long)blockIdx.x * tt;
    const int here = (int)(j.tokens - tok0 < tt ? j.tokens - tok0 : tt);
    const int hq = j.q.heads, hk = j.k.heads, heads = hq + hk + (PAGED ? j.v.heads : 0);
    const unsigned per_token = (unsigned)heads * pieces, total = per_token * here;
    const int turned = n / VE;

    // BATCH items a thread at a time, the first of them on their way while the angles are made
    struct Item { unsigned t, h, piece; };
    auto item = [&](unsigned it) {
        Item x;
        x.t = it / per_token;
        const unsigned r = it - x.t * per_token;
        x.h = r / pieces;
        x.piece = r - x.h * pieces;
        return x;
    };
    auto turns = [&](const Item& x) { return (int)x.piece < turned && (int)x.h < hq + hk; };
    auto first = [&](const Item& x) { return turns(x) && !j.adjacent ? VE * x.piece : 2 * VE * x.piece; };
    auto second = [&](const Item& x) { return turns(x) && !j.adjacent ? n + VE * x.piece : 2 * VE * x.piece + VE; };
    V a[BATCH], b[BATCH];
    auto fetch = [&](unsigned base) {
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const unsigned it = base + u * THREADS;
            if (it >= total) continue;
            const Item x = item(it);
            const bool q = (int)x.h < hq, k = !PAGED || (int)x.h < hq + hk;
            const Heads& from = q ? j.q : (k ? j.k : j.v);
            const T* src = (const T*)from.data + (tok0 + x.t) * from.token + (long)((int)x.h - (q ? 0 : (k ? hq : hq + hk))) * from.head;
            const int hi = second(x);
            a[u] = load_once<PAGED, V>(src + first(x));
            if (hi < j.dim) b[u] = load_once<PAGED, V>(src + hi);
        }
    };
    fetch(tid);

    if (PAGED && tid >= THREADS - MAX_TOKENS && tid - (THREADS - MAX_TOKENS) < here)
        find_place(j, c, tok0 + tid - (THREADS - MAX_TOKENS), &place[tid - (THREADS - MAX_TOKENS)]);
    for (int i = tid; i < here * n; i += THREADS) {
        const int t = i / n, p = i - t * n;
        int axis = 0;
#pragma unroll
        for (int a = 0; a < CB_ROTARY_MAX_AXES - 1; ++a) axis += a + 1 < j.axes && p >= j.end[a];
        // (whole turns go in float64: what is left is exact to float32)
        double turn = (double)j.positions[(tok0 + t) * j.pos_axes + axis] * j.turns[p];
        turn -= __builtin_rint(turn);
        float s, co;
        sincospif(2.0f * (float)turn, &s, &co);
        cs[i] = make_float2(co, j.inverse ? -s : s);
    }
    __syncthreads();
    if (PAGED && lengths != LENGTHS_LATER) {
        if (lengths == LENGTHS_FIRST) {
            if (blockIdx.x == 0) set_lengths(j, c, tid, THREADS);
        } else {
            // start is lengths itself: every workgroup has read it (above) before the last one writes it
            if (tid == 0) {
                int* counter = reinterpret_cast<int*>(c.scratch);
                last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
                if (last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (last) set_lengths(j, c, tid, THREADS);
        }
    }

    for (unsigned base = tid; base < total;) {
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const unsigned it = base + u * THREADS;
            if (it >= total) continue;
            const Item x = item(it);
            T* dst;
            if ((int)x.h < hq) {
                dst = (T*)j.q_out.data + (tok0 + x.t) * j.q_out.token + (long)x.h * j.q_out.head;
                if (PAGED && place[x.t].ignored) continue;
            } else if (!PAGED)
                dst = (T*)j.k_out.data + (tok0 + x.t) * j.k_out.token + (long)((int)x.h - hq) * j.k_out.head;
            else {
                const bool key = (int)x.h < hq + hk;
                if (place[x.t].row < 0) continue;
                dst = (T*)(key ? c.k : c.v) + place[x.t].row + (((long)((int)x.h - (key ? hq : hq + hk)) * c.dim) << c.page_shift);
            }
            if (turns(x)) {
                const float2* at = cs + x.t * n + x.piece * VE;
                V y, z;
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    if (!j.adjacent || VE == 1) {
                        const float p = widen(a[u].e[e]), q = widen(b[u].e[e]);
                        narrow(p * at[e].x - q * at[e].y, y.e[e]);
                        narrow(p * at[e].y + q * at[e].x, z.e[e]);
                    } else if ((e & 1) == 0) {
                        const int f = VE > 1 ? e + 1 : e;      // (there is one: VE is even here)
                        const float2 s = at[e / 2], w = at[VE / 2 + e / 2];
                        const float p = widen(a[u].e[e]), q = widen(a[u].e[f]), r = widen(b[u].e[e]), v = widen(b[u].e[f]);
                        narrow(p * s.x - q * s.y, y.e[e]);
                        narrow(p * s.y + q * s.x, y.e[f]);
                        narrow(r * w.x - v * w.y, z.e[e]);
                        narrow(r * w.y + v * w.x, z.e[f]);
                    }
                }
                a[u] = y;
                b[u] = z;
            }
            const int hi = second(x);
            store_once<PAGED>(a[u], dst + first(x));
            if (hi < j.dim) store_once<PAGED>(b[u], dst + hi);
        }
        base += BATCH * THREADS;
        if (base < total) fetch(base);
    }
    if (PAGED) {
        for (int i = tid; i < here * c.heads; i += THREADS) {
            const int t = i / c.heads;
            if (place[t].slot < 0 || place[t].ignored) continue;
            const long at = place[t].slot + (long)(i - t * c.heads) * c.capacity;
            if (c.weight) c.weight[at] = 0.0f;
            if (c.time) c.time[at] = place[t].time;
        }
    }
}

// Values of a vector: as many as 16 bytes hold, fewer where the pairs, a stride or an address do not divide into such
// vectors (one value at a time fits everything).
int vector_values(const RotaryJob& j)
{
    const int size = j.bf16 ? 2 : 4;
    int ve = 16 / size;
    const Heads* all[] = {&j.q, &j.q_out, &j.k, &j.k_out, &j.v};
    for (; ve > 1; ve /= 2) {
        bool fits = j.pairs % ve == 0;
        for (const Heads* h : all)
            fits = fits && (h->heads == 0 || !h->data ||
                            ((uintptr_t)h->data % (size * ve) == 0 && h->token % ve == 0 && h->head % ve == 0));
        if (fits) break;
    }
    return ve;
}

// Tokens of a workgroup: as many as its threads take in one batch and as it has angles for, as long as there are workgroups for
// every compute unit left.
int tokens_of_group(const RotaryJob& j, int pieces)
{
    const int items = (j.q.heads + j.k.heads + j.v.heads) * pieces, angles = j.pairs ? MAX_ANGLES / j.pairs : MAX_TOKENS;
    int tt = BATCH * THREADS / items;
    tt = tt < angles ? tt : angles;
    tt = tt < 1 ? 1 : (tt > MAX_TOKENS ? MAX_TOKENS : tt);
    while (tt > 1 && j.tokens / tt < 4L * device_units()) tt /= 2;
    return tt;
}

template <bool PAGED>
hipError_t launch(const RotaryJob& j, const Cache& c, int lengths, hipStream_t st)
{
    const int ve = vector_values(j), pieces = (j.dim + 2 * ve - 1) / (2 * ve), tt = tokens_of_group(j, pieces);
    const dim3 grid((unsigned)((j.tokens + tt - 1) / tt)), block(THREADS);
    if (lengths == LENGTHS_LAST && grid.x > 64) lengths = LENGTHS_LATER;
#define CB_ROTARY(type, n) hipLaunchKernelGGL((rotary_kernel<type, n, PAGED>), grid, block, 0, st, j, c, tt, pieces, lengths)
    if (j.bf16) {
        if (ve == 8) CB_ROTARY(uint16_t, 8);
        else if (ve == 4) CB_ROTARY(uint16_t, 4);
        else if (ve == 2) CB_ROTARY(uint16_t, 2);
        else CB_ROTARY(uint16_t, 1);
    } else {
        if (ve == 4) CB_ROTARY(float, 4);
        else if (ve == 2) CB_ROTARY(float, 2);
        else CB_ROTARY(float, 1);
    }
#undef CB_ROTARY
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !PAGED || lengths != LENGTHS_LATER) return e;
    hipLaunchKernelGGL(lengths_kernel, dim3((c.seqs + THREADS - 1) / THREADS), block, 0, st, j, c);
    return hipGetLastError();
}

}  // namespace

// (a launch has fewer than 2^32 threads: at most MOST_TOKENS tokens with a workgroup each)
hipError_t launch_rotate(const RotaryJob& all, hipStream_t st)
{
    const long size = all.bf16 ? 2 : 4;
    for (long at = 0; at < all.tokens; at += MOST_TOKENS) {
        RotaryJob j = all;
        j.tokens = all.tokens - at < MOST_TOKENS ? all.tokens - at : MOST_TOKENS;
        j.positions += at * j.pos_axes;
        for (Heads* h : {&j.q, &j.q_out, &j.k, &j.k_out}) h->data = (const char*)h->data + at * h->token * size;
        const hipError_t e = launch<false>(j, Cache(), LENGTHS_LATER, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// lengths of the cache are written by the first workgroup where start is another array; where it is the same one, by the
// workgroup that comes last of up to 64, behind which a launch of its own is cheaper (the workgroups' additions to one
// counter take about 11 ns each, one after the other)
hipError_t launch_append(const RotaryJob& j, const Cache& c, hipStream_t st)
{
    if (j.tokens == 0) {
        hipLaunchKernelGGL(lengths_kernel, dim3((c.seqs + THREADS - 1) / THREADS), dim3(THREADS), 0, st, j, c);
        return hipGetLastError();
    }
    return launch<true>(j, c, j.start == c.lengths ? LENGTHS_LAST : LENGTHS_FIRST, st);
}

}  // namespace cb
