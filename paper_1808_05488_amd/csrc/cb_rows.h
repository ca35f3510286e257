// What kernels that stream rows of heads past a token's angles share: vectors of values, loads and stores that pass the caches by, angles.
#pragma once
#include "cb_tokens.h"

namespace cb {

namespace {

template <typename T, int VE> struct alignas(sizeof(T) * VE) Vec { T e[VE]; };

template <int BYTES> struct Word;
template <> struct Word<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <> struct Word<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<2> { typedef uint16_t type; };
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

// Cosine and sine of a token's pair.  (Whole turns go in float64: what is left is exact to float32.)
__device__ __forceinline__ float2 angle_of(const RotaryJob& j, long token, int pair)
{
    int axis = 0;
#pragma unroll
    for (int a = 0; a < CB_ROTARY_MAX_AXES - 1; ++a) axis += a + 1 < j.axes && pair >= j.end[a];
    double turn = (double)j.positions[token * j.pos_axes + axis] * j.turns[pair];
    turn -= __builtin_rint(turn);
    float s, co;
    sincospif(2.0f * (float)turn, &s, &co);
    return make_float2(co, j.inverse ? -s : s);
}

// Two vectors of a head's pairs, turned by the angles at `at`.  HALVES: first values in one, second ones in the other; adjacent pairs: vector
// after vector.  (One value a vector is the same in both.)
template <int VE> __device__ __forceinline__ void turn(const float2* at, bool adjacent, float (&a)[VE], float (&b)[VE])
{
    float y[VE], z[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        if (!adjacent || VE == 1) {
            y[e] = a[e] * at[e].x - b[e] * at[e].y;
            z[e] = a[e] * at[e].y + b[e] * at[e].x;
        } else if ((e & 1) == 0) {
            const int f = VE > 1 ? e + 1 : e;                  // (there is one: VE is even here)
            const float2 s = at[e / 2], w = at[VE / 2 + e / 2];
            y[e] = a[e] * s.x - a[f] * s.y;
            y[f] = a[e] * s.y + a[f] * s.x;
            z[e] = b[e] * w.x - b[f] * w.y;
            z[f] = b[e] * w.y + b[f] * w.x;
        }
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) { a[e] = y[e]; b[e] = z[e]; }
}

// lengths after the call: start + rows, as far as there are such rows and room
__device__ __forceinline__ void set_lengths(const RotaryJob& j, const Cache& c, int first, int step)
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

// Values of a vector: as many as 16 bytes hold, fewer where the pairs, a stride or an address do not divide into such
// vectors (one value at a time fits everything).
template <int N> int vector_values(bool bf16, int pairs, const Heads* const (&all)[N])
{
    const int size = bf16 ? 2 : 4;
    int ve = 16 / size;
    for (; ve > 1; ve /= 2) {
        bool fits = pairs % ve == 0;
        for (const Heads* h : all)
            fits = fits && (h->heads == 0 || !h->data ||
                            ((uintptr_t)h->data % (size * ve) == 0 && h->token % ve == 0 && h->head % ve == 0));
        if (fits) break;
    }
    return ve;
}

}  // namespace

}  // namespace cb
