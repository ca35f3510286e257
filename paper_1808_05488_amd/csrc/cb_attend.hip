// Attention of one new token per sequence over a paged cache (cb_attend.h): over all its tokens, in the values' type; the weights that it adds up; what is
// launched for which cache.
#include "cb_attend.h"

namespace cb {

namespace {

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

hipError_t launch_attend_all(const AttendArgs& a, int groups, hipStream_t st)
{
    return a.c.bf16 ? launch_attend_as<uint16_t, uint16_t, false>(a, groups, st) : launch_attend_as<float, float, false>(a, groups, st);
}

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
    a.chosen = j.chosen;
    a.count = j.count;
    a.budget = j.budget;
    a.out_aligned = (uintptr_t)j.out.data % 16 == 0 && j.out.token % align == 0 && j.out.head % align == 0;
    // one workgroup a compute unit, no more than there can be tiles
    const long slots = j.chosen && j.budget < c.max_pages ? (long)j.budget << c.page_shift : c.capacity;
    const long most = (long)c.seqs * c.heads * a.blocks * (slots / (c.bf16 || c.e4m3 ? 32 : 16) + 1);
    const long want = device_units();
    const int groups = (int)(most < want ? most : (want < MAX_GROUPS ? want : MAX_GROUPS));
    const hipError_t e = j.chosen ? (c.e4m3 ? launch_attend_chosen_bytes(a, groups, st) : launch_attend_chosen(a, groups, st))
                                  : (c.e4m3 ? launch_attend_bytes(a, groups, st) : launch_attend_all(a, groups, st));
    if (e != hipSuccess || !j.accumulate) return e;
    hipLaunchKernelGGL(weight_kernel, dim3((c.capacity + 1023) / 1024, c.heads, c.seqs), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace cb
