// Products with 4-bit weights in groups for many rows: the 256 x 256 tile, whose sums are in units of the group's scale (the
// kernel is in quik_w4g_tiles_device.h).
#include "quik_w4g_tiles_device.h"

namespace quik {

hipError_t launch_w4g_tiles256(const W4gArgs& a, hipStream_t stream) {
    if (a.group != 128 || a.ids || a.glu) return hipErrorInvalidValue;
    return a.bf16 ? launch_tiles<Bf16, 128, 8, 4, 2, 4, 1, 2, 2, false>(a, stream)
                  : launch_tiles<Half, 128, 8, 4, 2, 4, 1, 2, 2, false>(a, stream);
}

}  // namespace quik
