// A layer of experts around its products (quik_w4g.hip): which experts a token goes to, its rows ordered by expert, and
// the weighted sum of what comes back.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "quik.h"
#include "quik_w4g.h"

namespace quik {

namespace {

using namespace w4g;

// ---- router: a wave per token, expert 64 i + lane in register i, all of it in 64 bits

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
// the largest value of the wave and the lowest index that has it
__device__ __forceinline__ void wave_top(double& v, int& i) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const double ov = __shfl_xor(v, d);
        const int oi = __shfl_xor(i, d);
        if (ov > v || (ov == v && oi < i)) { v = ov; i = oi; }
    }
}

__device__ __forceinline__ float load_logit(const void* p, int type, size_t at) {
    if (type == QUIK_F32) return static_cast<const float*>(p)[at];
    return type == QUIK_F16 ? Half::load(p, at) : Bf16::load(p, at);
}

template <int VPL>
__global__ __launch_bounds__(256) void moe_route_kernel(MoeRouteArgs a) {
    const int lane = threadIdx.x & 63;
    const int t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= a.T) return;
    const double kOut = -INFINITY;
    double score[VPL], choice[VPL];
    double top = kOut;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = i * 64 + lane;
        const float l = e < a.E ? load_logit(a.logits, a.type, (size_t)t * a.ldl + e) : -INFINITY;
        score[i] = l == l ? (double)l : kOut;            // (NaN: out)
        if (score[i] > top) top = score[i];
    }
    int none = 0;
    wave_top(top, none);
    double total = 0.0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const bool out = score[i] == kOut;
        if (a.sigmoid) score[i] = 1.0 / (1.0 + exp(-score[i]));
        else score[i] = out ? 0.0 : score[i] == top ? 1.0 : exp(score[i] - top);
        total += score[i];
        choice[i] = out ? kOut : score[i];
    }
    if (!a.sigmoid) total = wave_sum(total);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = i * 64 + lane;
        const bool out = choice[i] == kOut;
        if (!a.sigmoid && !out) score[i] /= total;
        const double c = score[i] + (a.bias && e < a.E ? (double)a.bias[e] : 0.0);
        choice[i] = out || c != c ? kOut : c;
    }
    if (a.groups > 1) {
        const int size = a.E / a.groups;
        double mine = kOut;                              // lane g: the score of group g
        for (int g = 0; g < a.groups; ++g) {
            double sum = kOut, used = INFINITY;
            int used_e = -1;
            for (int k = 0; k < a.group_top; ++k) {
                double v = kOut;
                int at = INT32_MAX;
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    const int e = i * 64 + lane;
                    if (e < g * size || e >= (g + 1) * size) continue;
                    if (choice[i] > used || (choice[i] == used && e <= used_e)) continue;
                    if (choice[i] > v || (choice[i] == v && e < at)) { v = choice[i]; at = e; }
                }
                wave_top(v, at);
                if (v == kOut) break;
                sum = k ? sum + v : v;
                used = v;
                used_e = at;
            }
            if (lane == g) mine = sum;
        }
        unsigned long long kept = 0;
        for (int k = 0; k < a.topk_groups; ++k) {
            double v = mine;
            int at = lane;
            wave_top(v, at);
            if (v == kOut) break;
            kept |= 1ull << at;
            if (lane == at) mine = kOut;
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int e = i * 64 + lane;
            if (e < a.E && !((kept >> (e / size)) & 1)) choice[i] = kOut;
        }
    }
    double sum = 0.0, mine = 0.0;                        // lane j: the score of slot j
    int id = -1;
    for (int j = 0; j < a.top_k; ++j) {
        double v = kOut;
        int at = INT32_MAX;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (choice[i] > v) { v = choice[i]; at = i * 64 + lane; }
        wave_top(v, at);
        if (v == kOut) break;
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (at == i * 64 + lane) { s = score[i]; choice[i] = kOut; }
        s = __shfl(s, at & 63);
        sum += s;
        if (lane == j) { mine = s; id = at; }
    }
    if (lane < a.top_k) {
        if (a.renormalize) mine = sum > 0.0 ? mine / sum : 0.0;
        a.ids[(size_t)t * a.top_k + lane] = id;
        a.weights[(size_t)t * a.top_k + lane] = (float)(mine * a.scale);
    }
}

// ---- plan: a workgroup per expert, and one for the rows of none.  Each counts the rows of the experts before its own and
// then lists its own in ascending order: no workgroup waits for another, and the order does not depend on timing.

constexpr int kPlanThreads = 1024;

__global__ __launch_bounds__(kPlanThreads) void moe_plan_kernel(const int32_t* ids, int rows, int experts, int32_t* plan) {
    __shared__ int part[kPlanThreads / 64 + 1];
    asm volatile("" ::: "v63");                          // a whole share of the register file (see quik_gemm.hip)
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, me = blockIdx.x;
    auto bucket = [&](int r) {
        const int e = ids[r];
        return e >= 0 && e < experts ? e : experts;
    };
    int less = 0;
    for (int r = tid; r < rows; r += kPlanThreads) less += bucket(r) < me;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) less += __shfl_xor(less, d);
    if (lane == 0) part[wave] = less;
    __syncthreads();
    less = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) less += part[w];
    if (tid == 0) {
        plan[me] = less;
        if (me == experts) plan[experts + 1] = rows;
    }
    int32_t* const list = plan + experts + 2;
    int at = less;
    for (int r0 = 0; r0 < rows; r0 += kPlanThreads) {
        const int r = r0 + tid;
        const bool mine = r < rows && bucket(r) == me;
        const unsigned long long m = __ballot(mine);
        __syncthreads();
        if (lane == 0) part[wave] = __popcll(m);
        __syncthreads();
        int before = 0, all = 0;
        for (int w = 0; w < kPlanThreads / 64; ++w) {
            const int c = part[w];
            before += w < wave ? c : 0;
            all += c;
        }
        if (mine) list[at + before + __popcll(m & ((1ull << lane) - 1))] = r;
        at += all;
    }
}

// ---- the slots' weighted sum, in slot order and fp32; slots of no expert take no part
template <typename TY>
__global__ __launch_bounds__(256) void moe_combine_kernel(const float* stage, const int32_t* ids, const float* weights, int T, int top_k,
                                                          int experts, int width, void* y, int ldy) {
    const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= (size_t)T * width) return;
    const size_t t = at / width, n = at % width;
    float v = 0.0f;
    for (int j = 0; j < top_k; ++j) {
        const size_t r = t * top_k + j;
        if (ids[r] >= 0 && ids[r] < experts) v = __builtin_fmaf(weights[r], stage[r * width + n], v);
    }
    static_cast<uint16_t*>(y)[t * ldy + n] = TY::round(v);
}

}  // namespace

hipError_t launch_moe_route(const MoeRouteArgs& a, hipStream_t stream) {
    const dim3 grid((a.T + 3) / 4), threads(256);
    const int vpl = (a.E + 63) / 64;
    if (vpl <= 1) hipLaunchKernelGGL(moe_route_kernel<1>, grid, threads, 0, stream, a);
    else if (vpl <= 2) hipLaunchKernelGGL(moe_route_kernel<2>, grid, threads, 0, stream, a);
    else if (vpl <= 4) hipLaunchKernelGGL(moe_route_kernel<4>, grid, threads, 0, stream, a);
    else if (vpl <= 8) hipLaunchKernelGGL(moe_route_kernel<8>, grid, threads, 0, stream, a);
    else hipLaunchKernelGGL(moe_route_kernel<16>, grid, threads, 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_moe_plan(const int32_t* ids, int rows, int experts, int32_t* plan, hipStream_t stream) {
    hipLaunchKernelGGL(moe_plan_kernel, dim3(experts + 1), dim3(kPlanThreads), 0, stream, ids, rows, experts, plan);
    return hipGetLastError();
}

hipError_t launch_moe_combine(const float* stage, const int32_t* ids, const float* weights, int T, int top_k, int experts,
                              int width, int bf16, void* y, int ldy, hipStream_t stream) {
    const dim3 grid((unsigned)(((size_t)T * width + 255) / 256)), threads(256);
    if (bf16) hipLaunchKernelGGL(moe_combine_kernel<Bf16>, grid, threads, 0, stream, stage, ids, weights, T, top_k, experts, width, y, ldy);
    else hipLaunchKernelGGL(moe_combine_kernel<Half>, grid, threads, 0, stream, stage, ids, weights, T, top_k, experts, width, y, ldy);
    return hipGetLastError();
}

}  // namespace quik
