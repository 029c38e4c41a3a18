// Which rows a workgroup of a w4g product has, and how it reads them.  Private to the shared library.
#pragma once
#include "quik_gemm_device.h"
#include "quik_w4g.h"

namespace quik {
namespace w4g {

constexpr uint32_t kRange = 0xFFFF0000u, kBeyond = 0xFFFFF000u;   // of a descriptor over whatever x is; a copy of zeros

// (offsets are checked against the matrix on the host, or made of indices that are)
__device__ __forceinline__ gemm_dev::v4i whole_rsrc(const void* p) {
    const uint64_t q = (uint64_t)(uintptr_t)p;
    gemm_dev::v4i r = gemm_dev::v4i{(int)(uint32_t)q, (int)(uint32_t)(q >> 32), (int)kRange, 0x00020000};
#pragma unroll
    for (int i = 0; i < 3; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
    return r;
}

struct RowSource {
    int expert;                      // -1: none, the rows are zeros
    int first, count;                // rows first .. first + count - 1 of the list, or of the output
    bool listed;                     // through the plan's list
};

// The rows of block b of a plan, bm to a block: the blocks of an expert's rows follow each other, then those of no expert;
// count 0 beyond the last.  Every wave finds the same, 64 experts at a time, one to a lane.  (At most 1024 experts.)
__device__ __forceinline__ RowSource planned_rows(const int32_t* plan, int experts, int b, int bm) {
    const int lane = threadIdx.x & 63;
    RowSource r{-1, 0, 0, true};
    for (int e0 = 0; e0 <= experts; e0 += 64) {
        const int e = e0 + lane;
        const int at = e <= experts ? plan[e] : 0, end = e <= experts ? plan[e + 1] : 0, mine = (end - at + bm - 1) / bm;
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        const unsigned long long here = __ballot(b >= upto - mine && b < upto);
        if (here) {
            const int l = __ffsll(here) - 1;
            const int first = __shfl(at, l) + (b - __shfl(upto - mine, l)) * bm;
            r.expert = e0 + l < experts ? e0 + l : -1;
            r.first = first;
            r.count = min(bm, __shfl(end, l) - first);
            break;
        }
        b -= __shfl(upto, 63);
    }
    r.expert = __builtin_amdgcn_readfirstlane(r.expert);
    r.first = __builtin_amdgcn_readfirstlane(r.first);
    r.count = __builtin_amdgcn_readfirstlane(r.count);
    return r;
}

}  // namespace w4g
}  // namespace quik
