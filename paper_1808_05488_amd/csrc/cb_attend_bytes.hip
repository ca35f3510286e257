// Attention of one new token per sequence (cb_attend.h): over all tokens of a cache in 8 bits.
#include "cb_attend.h"

namespace cb {

hipError_t launch_attend_bytes(const AttendArgs& a, int groups, hipStream_t st)
{
    return a.c.bf16 ? launch_attend_as<uint8_t, uint16_t, false>(a, groups, st) : launch_attend_as<uint8_t, float, false>(a, groups, st);
}

}  // namespace cb
