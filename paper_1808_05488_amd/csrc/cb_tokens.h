// Internal launcher interface of the token operators (rotary positions, paged cache, attention of one token, eviction): what the ABI
// layer cb_tokens.hip has checked, as plain values.  Every launcher enqueues on the given stream and returns the launch's hipError_t.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/cbconv.h"

namespace cb {

// A cb_heads with its element type left open.
struct Heads {
    const void* data = nullptr;
    long token = 0, head = 0;      // strides, in values
    int heads = 0;
};

// A cb_cache, checked, with what follows from it.
struct Cache {
    int seqs, heads, dim, page_shift, max_pages, n_pages, capacity, bf16;
    void *k, *v;
    const int32_t* table;
    int32_t* lengths;
    float* weight;
    int32_t* time;
    char* scratch;
};

// The scratch buffer: counters that every call leaves at zero, at places that depend on no size (caches share a buffer), then
// room that calls fill before they read it.
//   append:  counter 0: workgroups that have read the lengths
//   attend:  counter ATTEND_COUNTERS + w: workgroups that have written their part of the (sequence, key head, block of query
//            heads) whose first part is workgroup w's last one
constexpr int ATTEND_ROWS = 16;            // query heads of a block
constexpr int MAX_GROUPS = 1024;           // workgroups of the attention's launch at most
constexpr int ATTEND_COUNTERS = 64;
constexpr int COUNTER_BYTES = (ATTEND_COUNTERS + MAX_GROUPS) * 4;

struct ScratchPlan {
    size_t parts, sums, scores, moves, total;
};
ScratchPlan scratch_plan(const Cache& c, int q_heads);

struct RotaryJob {
    double turns[CB_ROTARY_MAX_PAIRS];
    int pairs, axes;               // 0 pairs: nothing turns
    int end[CB_ROTARY_MAX_AXES];   // first pair behind each axis
    int adjacent, inverse;
    int pos_axes;                  // integers a token in positions
    int dim, bf16;
    long tokens;
    const int32_t* positions;
    Heads q, q_out, k, k_out, v;   // no heads: not there; k_out: none where k and v go into a cache
    // append
    const int32_t *offsets, *start;
};
constexpr long MOST_TOKENS = (1L << 24) - 1;      // of a launch
hipError_t launch_rotate(const RotaryJob& j, hipStream_t st);
hipError_t launch_append(const RotaryJob& j, const Cache& c, hipStream_t st);

struct AttendJob {
    Heads q, out;
    float* lse;
    float scale, softcap, decay;
    int accumulate;
};
bool attend_fits(const Cache& c, int q_heads);      // its work can be counted in 32 bits
hipError_t launch_attend(const AttendJob& j, const Cache& c, hipStream_t st);

struct EvictJob {
    int budget, window;
    const float* weight_in;
    const int32_t *time_in, *lengths_in;
};
hipError_t launch_evict(const EvictJob& j, const Cache& c, hipStream_t st);

// Compute units of the current device.
int device_units();

#if defined(__HIPCC__)
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
// to the nearest, ties to even; what is not a number stays so
__device__ __forceinline__ void narrow(float f, float& to) { to = f; }
__device__ __forceinline__ void narrow(float f, uint16_t& to)
{
    __bf16 b = (__bf16)f;
    to = __builtin_bit_cast(uint16_t, b);
}
// Sum over the lanes up to this one, without LDS: within rows of 16 lanes, then across them.  All lanes take part.
__device__ __forceinline__ int wave_scan(int first)
{
    uint32_t v = (uint32_t)first;
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false);      // row_shr:1, 2, 4, 8
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);      // lane 15 of a row to the next, rows 1 and 3
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);      // lane 31 to rows 2 and 3
    return (int)v;
}
// The largest of all lanes, in every lane.
__device__ __forceinline__ int wave_max(int v)
{
    v = max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x111, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x112, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x114, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x118, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x142, 0xa, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ uint32_t wave_max_unsigned(uint32_t v) { return (uint32_t)wave_max((int)(v ^ 0x80000000u)) ^ 0x80000000u; }
// The sum of all lanes, in a fixed order, in every lane.
__device__ __forceinline__ float wave_sum(float v)
{
    auto add = [](float a, int b) { return a + __uint_as_float((uint32_t)b); };
    v = add(v, __builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x111, 0xf, 0xf, false));
    v = add(v, __builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x112, 0xf, 0xf, false));
    v = add(v, __builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x114, 0xf, 0xf, false));
    v = add(v, __builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x118, 0xf, 0xf, false));
    v = add(v, __builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x142, 0xa, 0xf, false));
    v = add(v, __builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x143, 0xc, 0xf, false));
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}
// The largest of all lanes, none of which is not a number, in every lane.
__device__ __forceinline__ float wave_max(float v)
{
    const uint32_t b = __float_as_uint(v), m = wave_max_unsigned(b & 0x80000000u ? ~b : b | 0x80000000u);
    return __uint_as_float(m & 0x80000000u ? m & 0x7FFFFFFFu : ~m);
}
// Length of a sequence, whatever the array holds.
__device__ __forceinline__ int clamp_length(int n, int capacity) { return n < 0 ? 0 : (n > capacity ? capacity : n); }
#endif

}  // namespace cb
