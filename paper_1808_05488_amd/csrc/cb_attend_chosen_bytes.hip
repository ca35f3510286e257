// Attention of one new token per sequence (cb_attend.h): over chosen pages of a cache in 8 bits.
#include "cb_attend.h"

namespace cb {

hipError_t launch_attend_chosen_bytes(const AttendArgs& a, int groups, hipStream_t st)
{
    return a.c.bf16 ? launch_attend_as<uint8_t, uint16_t, true>(a, groups, st) : launch_attend_as<uint8_t, float, true>(a, groups, st);
}

}  // namespace cb
