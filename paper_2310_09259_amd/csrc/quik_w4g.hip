// Products with 4-bit weights in groups (layout: quik_w4g_device.h): y[t, n] = sum_k x[t, k] s[n, k / g] (q[n, k] -
// z[n, k / g]), for a dense layer and for the experts that a router chose.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "quik_gemm_device.h"
#include "quik_w4g.h"

namespace quik {

namespace {

using namespace w4g;

// ---- the weights, once: one thread per dword of codes, and per stored group

struct PackArgs {
    const uint8_t* w_q;
    int ldw;
    const uint16_t* w_scale;
    const int8_t* w_zero;
    int N, K, G, group, kg, glu, nt, kt;
    uint32_t* codes;
    uint16_t* scales;
    int8_t* zeros;
};

// channel l of block b, or -1
__device__ __forceinline__ int channel_of(int b, int l, int N, int glu) {
    if (!glu) return b * kBlock + l < N ? b * kBlock + l : -1;
    const int f = (b >> 1) * kBlock + l;
    return f < N / 2 ? f + (b & 1) * (N / 2) : -1;
}

__global__ __launch_bounds__(256) void pack_w4g_kernel(PackArgs a) {
    const int tiles = a.nt * a.kt;
    const size_t e = blockIdx.y;
    const int tile = blockIdx.x, b = tile / a.kt, kt = tile % a.kt;
    {
        const int lane = threadIdx.x >> 2, s = threadIdx.x & 3;
        const int n = channel_of(b, lane & 15, a.N, a.glu), k = kt * kCols + s * 32 + (lane >> 4) * 8;
        uint32_t in = 0;
        if (n >= 0 && k < a.K) in = *reinterpret_cast<const uint32_t*>(a.w_q + (e * a.N + n) * a.ldw + k / 2);
        in ^= 0x88888888u;                               // code + 8
        uint32_t out = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) out |= ((in >> (8 * i)) & 15u) << (4 * i) | ((in >> (8 * i + 4)) & 15u) << (4 * i + 16);
        a.codes[(e * tiles + tile) * (kTileBytes / 4) + threadIdx.x] = out;
    }
    const int per = kCols / a.kg;
    if ((int)threadIdx.x < kBlock * per) {
        const int n = channel_of(b, threadIdx.x / per, a.N, a.glu), k = kt * kCols + threadIdx.x % per * a.kg;
        const bool in = n >= 0 && k < a.K;
        const size_t from = in ? (e * a.N + n) * a.G + k / a.group : 0, to = (e * tiles + tile) * kBlock * per + threadIdx.x;
        a.scales[to] = in ? a.w_scale[from] : 0;
        if (a.w_zero) a.zeros[to] = in ? a.w_zero[from] : 0;
    }
}

// ---- sixteen rows at a time

struct RowSource {                   // what a workgroup's sixteen rows are
    int expert;                      // -1: none, the rows are zeros
    int first, count;                // rows first .. first + count - 1 of the list, or of the output
    bool listed;                     // through plan's list
};

// the sixteen rows of block b of a plan: blocks of an expert's rows follow each other, then those of no expert
__device__ __forceinline__ RowSource planned_rows(const int32_t* plan, int experts, int b, int bm) {
    RowSource r{-1, 0, 0, true};
    for (int e = 0; e <= experts; ++e) {
        const int at = plan[e], blocks = (plan[e + 1] - at + bm - 1) / bm;
        if (b < blocks) {
            r.expert = e < experts ? e : -1;
            r.first = at + b * bm;
            r.count = min(bm, plan[e + 1] - r.first);
            return r;
        }
        b -= blocks;
    }
    return r;
}

// Four waves split K; the wave's partial sums are added in wave order.  A group's sum of x (q - z) is exact in its
// operands (16-bit activations, integers of at most eight bits) and held in fp32, and the scale is applied to it in fp32.
template <typename TY, int KG>
__global__ __launch_bounds__(256) void w4g_rows_kernel(W4gArgs a) {
    constexpr int NW = 4, CB = 2, PER = kCols / KG;
    __shared__ float red[NW][CB][64][4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, g = lane >> 4;
    const int b0 = blockIdx.x * CB;

    RowSource src{0, (int)blockIdx.y * 16, min(16, a.rows - (int)blockIdx.y * 16), false};
    if (a.ids && a.plan) {
        src = planned_rows(a.plan, a.experts, blockIdx.y, 16);
        if (src.count == 0) return;
    } else if (a.ids) {
        const int e = a.ids[blockIdx.y];
        src = RowSource{e >= 0 && e < a.experts ? e : -1, (int)blockIdx.y, 1, false};
    }
    const int32_t* list = src.listed ? a.plan + a.experts + 2 + src.first : nullptr;

    v4f acc[CB] = {};
    if (src.expert >= 0) {
        const uint8_t* codes = a.w.codes + src.expert * a.w.codes_e;
        const uint16_t* scales = reinterpret_cast<const uint16_t*>(a.w.scales + src.expert * a.w.scales_e);
        const int8_t* zeros = a.w.zeros ? reinterpret_cast<const int8_t*>(a.w.zeros + src.expert * a.w.zeros_e) : nullptr;
        const bool row_ok = l16 < src.count;
        int row = row_ok ? (list ? list[l16] : src.first + l16) : 0;
        if (a.ids && !a.x_per_slot) row /= a.top_k;
        const uint16_t* x = static_cast<const uint16_t*>(a.x) + (size_t)row * a.ldx;
        const v4u ones = v4u{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
        for (int kt = a.w.kt * wave / NW; kt < a.w.kt * (wave + 1) / NW; ++kt) {
            v4u xa[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int k = kt * kCols + s * 32 + g * 8;
                xa[s] = row_ok && k < a.w.K ? *reinterpret_cast<const v4u*>(x + k) : v4u{0, 0, 0, 0};
            }
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                if (b0 + c >= a.w.nt) continue;
                const size_t tile = (size_t)(b0 + c) * a.w.kt + kt;
                const v4u w = *reinterpret_cast<const v4u*>(codes + tile * kTileBytes + lane * 16);
#pragma unroll
                for (int p = 0; p < PER; ++p) {
                    const size_t at = (tile * 16 + l16) * PER + p;
                    const float scale = (float)__builtin_bit_cast(_Float16, scales[at]);
                    const float zero = 8.0f + TY::kOffset + (zeros ? (float)zeros[at] : 0.0f);
                    v4f part = {}, sum = {};
#pragma unroll
                    for (int s = p * (4 / PER); s < (p + 1) * (4 / PER); ++s) {
                        v4u b;
#pragma unroll
                        for (int i = 0; i < 4; ++i) b[i] = ((w[s] >> (4 * i)) & 0x000F000Fu) | TY::kBits;
                        if constexpr (TY::kOffset > 1000.0f) {
                            const v2h z = v2h{(_Float16)zero, (_Float16)zero};
#pragma unroll
                            for (int i = 0; i < 4; ++i) b[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, (uint32_t)b[i]) - z);
                        } else {
                            sum = TY::mfma(xa[s], ones, sum);
                        }
                        part = TY::mfma(xa[s], b, part);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v = part[r];
                        if constexpr (TY::kOffset < 1000.0f) v = __builtin_fmaf(-zero, sum[r], v);
                        acc[c][r] = __builtin_fmaf(scale, v, acc[c][r]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) red[wave][c][lane][r] = acc[c][r];
    __syncthreads();
    // wave c finishes block c of the two, or wave 0 both halves of a pair
    if (wave >= (a.glu ? 1 : CB)) return;
    const int n = a.glu ? (b0 >> 1) * kBlock + l16 : (b0 + wave) * kBlock + l16;
    if (n >= a.width) return;
    const size_t bias_at = (size_t)(src.expert > 0 ? src.expert : 0) * a.w.N;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = 4 * g + r;
        if (i >= src.count) continue;
        float v[2] = {0.0f, 0.0f};
        for (int h = 0; h < (a.glu ? 2 : 1); ++h) {
            for (int w = 0; w < NW; ++w) v[h] += red[w][a.glu ? h : wave][lane][r];
            if (a.bias && src.expert >= 0) v[h] += TY::load(a.bias, bias_at + n + h * a.width);
        }
        if (a.glu) v[0] = silu_product(v[0], v[1]);
        const size_t row = list ? list[i] : src.first + i;
        if (src.expert < 0) v[0] = 0.0f;
        if (a.weights) a.stage[row * a.width + n] = v[0];
        else static_cast<uint16_t*>(a.y)[row * a.ldy + n] = TY::round(v[0]);
    }
}

}  // namespace

hipError_t launch_weight_pack_w4g(const void* w_q, int ldw, const void* w_scale, const void* w_zero, int N, int K, int group,
                                  int glu, int experts, void* w4, hipStream_t stream) {
    const Layout l = layout(N, K, group, w_zero != nullptr, glu != 0, experts);
    uint8_t* const base = static_cast<uint8_t*>(w4);
    PackArgs a{static_cast<const uint8_t*>(w_q), ldw, static_cast<const uint16_t*>(w_scale), static_cast<const int8_t*>(w_zero),
               N, K, group ? (K + group - 1) / group : 1, group ? group : K, l.kg, glu, l.nt, l.kt,
               reinterpret_cast<uint32_t*>(base), reinterpret_cast<uint16_t*>(base + l.scales_at),
               reinterpret_cast<int8_t*>(base + l.zeros_at)};
    hipLaunchKernelGGL(pack_w4g_kernel, dim3(l.nt * l.kt, experts), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_w4g(const W4gArgs& args, hipStream_t stream) {
    W4gArgs a = args;
    int blocks = (a.rows + 15) / 16;
    if (a.ids) {
        if (a.rows <= a.experts) a.plan = nullptr;       // a row at a time: hardly two share an expert
        else if (hipError_t rc = launch_moe_plan(a.ids, a.rows, a.experts, a.plan, stream); rc != hipSuccess) return rc;
        blocks = a.plan ? (a.rows + 15) / 16 + min(a.rows, a.experts + 1) : a.rows;
    }
    const dim3 grid((a.w.nt + 1) / 2, blocks), threads(256);
    switch (a.group + a.bf16) {
        case 32: hipLaunchKernelGGL((w4g_rows_kernel<Half, 32>), grid, threads, 0, stream, a); break;
        case 64: hipLaunchKernelGGL((w4g_rows_kernel<Half, 64>), grid, threads, 0, stream, a); break;
        case 128: hipLaunchKernelGGL((w4g_rows_kernel<Half, 128>), grid, threads, 0, stream, a); break;
        case 33: hipLaunchKernelGGL((w4g_rows_kernel<Bf16, 32>), grid, threads, 0, stream, a); break;
        case 65: hipLaunchKernelGGL((w4g_rows_kernel<Bf16, 64>), grid, threads, 0, stream, a); break;
        case 129: hipLaunchKernelGGL((w4g_rows_kernel<Bf16, 128>), grid, threads, 0, stream, a); break;
        default: return hipErrorInvalidValue;
    }
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess || !a.weights) return rc;
    return launch_moe_combine(a.stage, a.ids, a.weights, a.rows / a.top_k, a.top_k, a.experts, a.width, a.bf16, a.y, a.ldy, stream);
}

}  // namespace quik
