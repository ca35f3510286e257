// Attention of one new token per sequence (cb_attend.h): over chosen pages.
#include "cb_attend.h"

namespace cb {

hipError_t launch_attend_chosen(const AttendArgs& a, int groups, hipStream_t st)
{
    return a.c.bf16 ? launch_attend_as<uint16_t, uint16_t, true>(a, groups, st) : launch_attend_as<float, float, true>(a, groups, st);
}

}  // namespace cb
