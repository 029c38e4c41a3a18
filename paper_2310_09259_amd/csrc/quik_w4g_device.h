// 4-bit weights with a scale (and a zero point) per group of input columns: their layout in memory and how the kernels
// widen them.  Private to the shared library.
//
// The matrix [N, K] is cut into tiles of 16 channels x 128 columns.  A tile's codes are 1 KB, 16 bytes for each lane
// of a wave: dword s of lane 16 g + l holds the eight columns 32 s + 8 g .. + 7 of channel l, which is what the lane
// feeds to the s-th 16 x 16 x 32 matrix instruction of the tile.  A wave so loads a tile with one instruction, whole
// lines in order, and never moves a code between lanes.  Codes are stored unsigned (code + 8); in a dword, column 2 i
// sits in nibble i and column 2 i + 1 in nibble i + 4, so that (dword >> 4 i) & 0x000F000F is a pair of neighbours in
// the halves of a register.  Tiles lie channel block by channel block, the columns of a block in order:
//   codes   [E][NT][KT][1024 bytes]           NT = channel blocks, KT = ceil(K / 128)
//   scales  [E][NT][KT][16][128 / KG]  fp16   KG = columns of a stored group: 32, 64 or 128
//   zeros   [E][NT][KT][16][128 / KG]  int8   (only if there are any)
// Larger groups are stored as equal groups of 128.  Columns beyond K and channels beyond N hold the code 0, groups
// beyond K and channels beyond N the scale 0.  With paired halves (glu) block 2 i holds channels 16 i .. of the gates
// and block 2 i + 1 the same channels of the values: a wave that takes two blocks has both factors of an output.
#pragma once
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stddef.h>
#include <stdint.h>

namespace quik {
namespace w4g {

constexpr int kBlock = 16;           // channels of a tile
constexpr int kCols = 128;           // columns of a tile
constexpr int kTileBytes = 1024;

struct Layout {
    int nt, kt, kg;                  // channel blocks, tiles along K, columns of a stored group
    size_t codes, scales, zeros;     // bytes of one expert in each region
    size_t scales_at, zeros_at, total;   // regions, and the whole buffer, in bytes
};

inline size_t up16(size_t v) { return (v + 15) & ~size_t(15); }

inline Layout layout(int N, int K, int group, bool has_zero, bool glu, int experts) {
    Layout w;
    w.nt = glu ? 2 * ((N / 2 + kBlock - 1) / kBlock) : (N + kBlock - 1) / kBlock;
    w.kt = (K + kCols - 1) / kCols;
    w.kg = group == 32 || group == 64 ? group : kCols;
    const size_t tiles = (size_t)w.nt * w.kt, groups = tiles * kBlock * (kCols / w.kg);
    w.codes = tiles * kTileBytes;
    w.scales = groups * 2;
    w.zeros = has_zero ? groups : 0;
    w.scales_at = w.codes * experts;
    w.zeros_at = w.scales_at + up16(w.scales * experts);
    w.total = w.zeros_at + up16(w.zeros * experts);
    return w;
}

// what a kernel reads of it
struct Weights {
    const uint8_t* codes;
    const uint8_t* scales;
    const uint8_t* zeros;            // or null
    size_t codes_e, scales_e, zeros_e;   // bytes from one expert to the next
    int N, K, nt, kt;
};

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

// The 16-bit types of the activations.  kBits | code is a number whose last place is 1: kOffset + code, exactly, with
// kOffset = 1024 in fp16 and 128 in bf16.
struct Half {
    static constexpr uint32_t kBits = 0x64006400u;
    static constexpr float kOffset = 1024.0f;
    static __device__ __forceinline__ v4f mfma(v4u a, v4u b, v4f c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float load(const void* p, size_t i) { return (float)static_cast<const _Float16*>(p)[i]; }
    static __device__ __forceinline__ uint16_t round(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};
struct Bf16 {
    static constexpr uint32_t kBits = 0x43004300u;
    static constexpr float kOffset = 128.0f;
    static __device__ __forceinline__ v4f mfma(v4u a, v4u b, v4f c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float load(const void* p, size_t i) { return (float)static_cast<const __bf16*>(p)[i]; }
    static __device__ __forceinline__ uint16_t round(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
};

// gate * sigmoid(gate) * value: v_exp_f32 and v_rcp_f32 (1 ulp each) beside a result rounded to 16 bits.  For a gate
// below -88 the exponential is infinite and the quotient -0, the limit.
__device__ __forceinline__ float silu_product(float gate, float value) {
    return gate * __builtin_amdgcn_rcpf(1.0f + __expf(-gate)) * value;
}

}  // namespace w4g
}  // namespace quik
