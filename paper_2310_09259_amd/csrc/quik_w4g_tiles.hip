// Products with 4-bit weights in groups for many rows: the tiles whose sums over a group have registers of their own (the
// kernel is in quik_w4g_tiles_device.h).
#include "quik_w4g_tiles_device.h"

namespace quik {

namespace {

template <typename TY, int KG>
hipError_t dispatch(const W4gArgs& a, int form, hipStream_t stream) {
    switch (form) {
        case kW4gTile32x128: return launch_tiles<TY, KG, 2, 2, 1, 4, 2, 4, 2, true>(a, stream);
        case kW4gTile64x128: return launch_tiles<TY, KG, 4, 2, 1, 4, 2, 3, 2, true>(a, stream);
        case kW4gTile128x128: return launch_tiles<TY, KG, 4, 2, 2, 4, 1, 3, 2, true>(a, stream);
        case kW4gTile256x128: return launch_tiles<TY, KG, 8, 2, 2, 4, 1, 2, 2, true>(a, stream);
        case kW4gTile32x128Small: return launch_tiles<TY, KG, 2, 2, 1, 4, 1, 2, 4, true>(a, stream);
        case kW4gTile64x128Small: return launch_tiles<TY, KG, 4, 2, 1, 4, 1, 2, KG == 128 ? 3 : 2, true>(a, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_w4g_tiles(const W4gArgs& a, int form, hipStream_t stream) {
    if (form == kW4gTile256x256) return launch_w4g_tiles256(a, stream);
    switch (a.group + a.bf16) {
        case 32: return dispatch<Half, 32>(a, form, stream);
        case 64: return dispatch<Half, 64>(a, form, stream);
        case 128: return dispatch<Half, 128>(a, form, stream);
        case 33: return dispatch<Bf16, 32>(a, form, stream);
        case 65: return dispatch<Bf16, 64>(a, form, stream);
        case 129: return dispatch<Bf16, 128>(a, form, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace quik
