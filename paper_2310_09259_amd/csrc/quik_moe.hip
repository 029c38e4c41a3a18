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

// ---- router: a wave per token, expert 64 i + lane in register i.
//
// What bounds it: the chain of reductions over the wave, some ten of them one behind the other, and for one token the
// latency of its logits; the bytes are nothing.  So maxima and sums go through the lanes' data paths (six vector
// instructions, no trip to LDS), and scores are computed in fp32.  Choices are told apart as float64 tells them: a token two
// of whose chosen ones, or any one left and the last one chosen, or groups next to the border lie within the error of the fp32
// scores of each other, or one of whose chosen scores is below 2^-100, goes through the same in float64.  Four groups of experts are reduced side by
// side.  4096 tokens and 256 experts in eight groups: 33 us all in float64, with shuffles through LDS; 24.9 one group after
// another; 20 to 24 as it is, by the tokens that go through float64 (for one token 10.4 and 9.5).  These are for logits of a
// standard deviation of 1.5; the bound is one of the largest score, and scores near 0 or 1 lie close together: over 256 experts
// without groups 9.6 us at 1.5, 14.7 at 8.

template <int CTRL, int ROWS> __device__ __forceinline__ float lane_move(float v) {
    const int i = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CTRL, ROWS, 0xF, false));
}
template <int CTRL, int ROWS> __device__ __forceinline__ double lane_move(double v) {
    const int2 i = __builtin_bit_cast(int2, v);
    return __builtin_bit_cast(double, make_int2(__builtin_amdgcn_update_dpp(i.x, i.x, CTRL, ROWS, 0xF, false),
                                                __builtin_amdgcn_update_dpp(i.y, i.y, CTRL, ROWS, 0xF, false)));
}
__device__ __forceinline__ float of_lane(float v, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
__device__ __forceinline__ double of_lane(double v, int lane) {
    const int2 i = __builtin_bit_cast(int2, v);
    return __builtin_bit_cast(double, make_int2(__builtin_amdgcn_readlane(i.x, lane), __builtin_amdgcn_readlane(i.y, lane)));
}
// over all 64 lanes: shifts by 1, 2, 4, 8 inside rows of 16, then the last lanes of rows to the next ones; lane 63 has it
template <typename F> __device__ __forceinline__ F wave_max(F v) {
    v = fmax(v, lane_move<0x111, 0xF>(v));
    v = fmax(v, lane_move<0x112, 0xF>(v));
    v = fmax(v, lane_move<0x114, 0xF>(v));
    v = fmax(v, lane_move<0x118, 0xF>(v));
    v = fmax(v, lane_move<0x142, 0xA>(v));
    v = fmax(v, lane_move<0x143, 0xC>(v));
    return of_lane(v, 63);
}
// of several values, step by step together
template <int N, typename F> __device__ __forceinline__ void wave_max_each(F (&v)[N]) {
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = fmax(v[q], lane_move<0x111, 0xF>(v[q]));
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = fmax(v[q], lane_move<0x112, 0xF>(v[q]));
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = fmax(v[q], lane_move<0x114, 0xF>(v[q]));
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = fmax(v[q], lane_move<0x118, 0xF>(v[q]));
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = fmax(v[q], lane_move<0x142, 0xA>(v[q]));
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = of_lane(fmax(v[q], lane_move<0x143, 0xC>(v[q])), 63);
}
template <typename F> __device__ __forceinline__ F wave_sum(F v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

__device__ __forceinline__ float load_logit(const void* p, int type, size_t at) {
    if (type == QUIK_F32) return static_cast<const float*>(p)[at];
    return type == QUIK_F16 ? Half::load(p, at) : Bf16::load(p, at);
}

// A token, with scores in F; logit: -infinity for an expert that takes no part.  float: false, with nothing written, if it may
// have told choices apart otherwise than double, or a chosen score is next to what fp32 cannot hold.
template <typename F, int VPL>
__device__ __forceinline__ bool route_token(const MoeRouteArgs& a, int t, const float (&logit)[VPL]) {
    constexpr bool EXACT = sizeof(F) == 8;
    constexpr F kOut = -INFINITY;
    const int lane = threadIdx.x & 63;
    F score[VPL], choice[VPL];
    float bias[VPL];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        top = fmaxf(top, logit[i]);
        bias[i] = a.bias && i * 64 + lane < a.E ? a.bias[i * 64 + lane] : 0.0f;
    }
    F largest = 1;                                       // of all scores, at least
    if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) score[i] = (F)1 / ((F)1 + exp(-(F)logit[i]));
    } else {
        top = wave_max(top);
        F part[VPL];
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            score[i] = logit[i] == -INFINITY ? (F)0 : logit[i] == top ? (F)1 : exp((F)logit[i] - (F)top);
            part[i] = score[i];
        }
#pragma unroll
        for (int d = 1; d < VPL; d *= 2)                 // (in pairs: four roundings of sixteen scores)
#pragma unroll
            for (int i = 0; i + d < VPL; i += 2 * d) part[i] += part[i + d];
        const F total = wave_sum(part[0]);
#pragma unroll
        for (int i = 0; i < VPL; ++i) score[i] /= total; // (nobody: NaN, and not looked at)
        largest = (F)1 / total;
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const F c = score[i] + (F)bias[i];
        choice[i] = logit[i] == -INFINITY || c != c ? kOut : c;
    }
    // How far apart two fp32 choices have to lie, in units of 2^-24.  The exponential is off by 4 of itself.  Sigmoid: times
    // 1 - s, and a unit each for the sum and the quotient, 6 s - 4 s^2 < 2.3 for a score, 4.6 for two.  Softmax, of the largest
    // score: 4.4 with the argument's rounding and one for the quotient, 10.8 for two, and what all have in common (it matters
    // beside a bias), 4.4 and ten roundings of the total: 25.2.  The choices' own rounding, and that of sums of such that are
    // not negative: one of each, or of every term, of the two.
    const F apart = a.sigmoid ? (F)0x1p-21 : (F)0x1p-19 * largest, rounding = (F)0x1p-22;
    bool sure = true;
    // the largest choice, its expert e (of equal ones the lowest), taken out of the list, its score, logit and bias;
    // -infinity: there is none
    auto pick = [&](int& e, F& s, float& l, float& b) {
        F mine = kOut;
        int at = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (choice[i] > mine) { mine = choice[i]; at = i; }
        const F v = wave_max(mine);
        const unsigned long long have = __ballot(mine == v && v > kOut);
        if (have == 0) return kOut;
        int from = __ffsll(have) - 1;
        if (have & (have - 1)) from = (int)-wave_max(mine == v ? -(float)(at * 64 + lane) : -INFINITY) & 63;
        at = __builtin_amdgcn_readlane(at, from);
        e = at * 64 + from;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (i == at) {
                s = of_lane(score[i], from);
                l = of_lane(logit[i], from);
                b = of_lane(bias[i], from);
                if (lane == from) choice[i] = kOut;
            }
        return v;
    };
    if (a.groups > 1) {
        const int size = a.E / a.groups;
        F mine = kOut;                                   // lane g: the score of group g
        constexpr int SIDE = VPL <= 4 ? 4 : 1;           // groups side by side: their reductions do not wait for each other
        for (int g = 0; g < a.groups; g += SIDE) {
            F in[SIDE][VPL], sum[SIDE];
#pragma unroll
            for (int q = 0; q < SIDE; ++q) {
                sum[q] = kOut;
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    const int e = i * 64 + lane;
                    in[q][i] = e >= (g + q) * size && e < (g + q + 1) * size ? choice[i] : kOut;   // (none beyond the last group)
                }
            }
            for (int k = 0; k < a.group_top; ++k) {
                F best[SIDE], v[SIDE];
                int at[SIDE];
#pragma unroll
                for (int q = 0; q < SIDE; ++q) {
                    best[q] = kOut;
                    at[q] = 0;
#pragma unroll
                    for (int i = 0; i < VPL; ++i)
                        if (in[q][i] > best[q]) { best[q] = in[q][i]; at[q] = i; }
                    v[q] = best[q];
                }
                wave_max_each<SIDE>(v);
                if (SIDE == 1 && v[0] == kOut) break;         // (nothing is left in it)
#pragma unroll
                for (int q = 0; q < SIDE; ++q) {
                    if (v[q] < 0 && v[q] > kOut) sure = false;                 // (a sum may be small beside what it is made of)
                    sum[q] = k && v[q] > kOut ? sum[q] + v[q] : k ? sum[q] : v[q];
                    const int from = __ffsll(__ballot(best[q] == v[q])) - 1;   // (one of equal ones: the sum is the same)
#pragma unroll
                    for (int i = 0; i < VPL; ++i)
                        if (lane == from && i == at[q]) in[q][i] = kOut;
                }
            }
#pragma unroll
            for (int q = 0; q < SIDE; ++q)
                if (lane == g + q) mine = sum[q];
        }
        unsigned long long kept = 0;
        F last = INFINITY;
        for (int k = 0; k <= a.topk_groups; ++k) {
            const F v = wave_max(mine);
            if (v == kOut) break;
            if (k == a.topk_groups) {                    // the first group that goes
                sure = sure && last - v > a.group_top * (apart + rounding * fabs(last));
                break;
            }
            const int at = __ffsll(__ballot(mine == v)) - 1;
            kept |= 1ull << at;
            last = v;
            if (lane == at) mine = kOut;
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int e = i * 64 + lane;
            if (e < a.E && !((kept >> (e / size)) & 1)) choice[i] = kOut;
        }
    }
    F sum = 0, mine = 0, last = INFINITY;                // mine, id: of slot `lane`
    float last_l = 0.0f, last_b = 0.0f;
    int id = -1;
    for (int j = 0; j < a.top_k; ++j) {
        int e = -1;
        F s = 0;
        float l = 0.0f, b = 0.0f;
        const F v = pick(e, s, l, b);
        if (v == kOut) break;
        if constexpr (!EXACT) {
            // a score that fp32 still holds all bits of, and weights are made of (in a sum of smaller ones they would vanish)
            sure = sure && s >= (F)0x1p-100;
            // equal for certain (the index decides), or apart for certain
            if (j > 0) sure = sure && ((l == last_l && b == last_b) || last - v > apart + rounding * fabs(last));
            if (!sure) break;
        }
        last = v;
        last_l = l;
        last_b = b;
        sum += s;
        if (lane == j) { mine = s; id = e; }
    }
    // the same of all that are left against the last one chosen: behind one that is equal to it another may be larger
    if (!EXACT && sure) {
        bool near = false;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            near = near || (choice[i] > kOut && !(logit[i] == last_l && bias[i] == last_b) && !(last - choice[i] > apart + rounding * fabs(last)));
        sure = __ballot(near) == 0;
    }
    if (!EXACT && !sure) return false;
    if (lane < a.top_k) {
        if (a.renormalize) mine = sum > 0 ? mine / sum : (F)0;
        a.ids[(size_t)t * a.top_k + lane] = id;
        a.weights[(size_t)t * a.top_k + lane] = id < 0 ? 0.0f : (float)(mine * (F)a.scale);   // (whatever the scale)
    }
    return true;
}

template <int VPL>
__global__ __launch_bounds__(256) void moe_route_kernel(MoeRouteArgs a) {
    asm volatile("" ::: "v127");                         // a whole share of the register file (see quik_gemm.hip)
    const int lane = threadIdx.x & 63;
    const int t = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (t >= a.T) return;
    float logit[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = i * 64 + lane;
        const float l = e < a.E ? load_logit(a.logits, a.type, (size_t)t * a.ldl + e) : -INFINITY;
        logit[i] = l == l ? l : -INFINITY;               // (NaN: out)
    }
    if (!route_token<float, VPL>(a, t, logit)) route_token<double, VPL>(a, t, logit);
}

// ---- plan: a workgroup per expert, and one for the rows of none.  Each counts the rows of the experts before its own and
// then lists its own in ascending order: no workgroup waits for another, and the order does not depend on timing.  A thread
// takes four rows at a time, and the first rounds' rows stay in registers between the passes.

constexpr int kPlanThreads = 1024, kPlanRound = kPlanThreads * 4, kPlanKept = 4;

__global__ __launch_bounds__(kPlanThreads) void moe_plan_kernel(const int32_t* ids, int rows, int experts, int32_t* plan) {
    asm volatile("" ::: "v63");                          // a whole share of the register file (see quik_gemm.hip)
    __shared__ int part[2][kPlanThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, me = blockIdx.x;
    const bool aligned = (reinterpret_cast<uintptr_t>(ids) & 15) == 0;
    auto buckets = [&](int r) {                          // of rows r .. r + 3; beyond the last, -1
        int4 v = make_int4(experts, experts, experts, experts);
        if (aligned && r + 3 < rows) {
            v = *reinterpret_cast<const int4*>(ids + r);
        } else {
            if (r < rows) v.x = ids[r];
            if (r + 1 < rows) v.y = ids[r + 1];
            if (r + 2 < rows) v.z = ids[r + 2];
            if (r + 3 < rows) v.w = ids[r + 3];
        }
        auto of = [&](int e, int row) { return row >= rows ? -1 : e >= 0 && e < experts ? e : experts; };
        return make_int4(of(v.x, r), of(v.y, r + 1), of(v.z, r + 2), of(v.w, r + 3));
    };
    int4 kept[kPlanKept];
    int less = 0;
    auto count = [&](int4 v) {
        auto one = [&](int e) { return e >= 0 && e < me; };
        less += one(v.x) + one(v.y) + one(v.z) + one(v.w);
    };
#pragma unroll
    for (int k = 0; k < kPlanKept; ++k) kept[k] = buckets(k * kPlanRound + tid * 4);
#pragma unroll
    for (int k = 0; k < kPlanKept; ++k) count(kept[k]);
    for (int r0 = kPlanKept * kPlanRound; r0 < rows; r0 += kPlanRound) count(buckets(r0 + tid * 4));
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) less += __shfl_xor(less, d);
    if (lane == 0) part[1][wave] = less;
    __syncthreads();
    int at = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) at += part[1][w];
    if (tid == 0) {
        plan[me] = at;
        if (me == experts) plan[experts + 1] = rows;
    }
    int32_t* const list = plan + experts + 2;
    auto place = [&](int4 v, int r, int round) {
        const int own = (v.x == me) + (v.y == me) + (v.z == me) + (v.w == me);
        int upto = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 63) part[round & 1][wave] = upto;
        __syncthreads();                                 // (the other half is written in the next round, behind this barrier)
        int to = at + upto - own;
        for (int w = 0; w < kPlanThreads / 64; ++w) {
            const int c = part[round & 1][w];
            to += w < wave ? c : 0;
            at += c;
        }
        if (v.x == me) list[to++] = r;
        if (v.y == me) list[to++] = r + 1;
        if (v.z == me) list[to++] = r + 2;
        if (v.w == me) list[to++] = r + 3;
    };
    int round = 0;
#pragma unroll
    for (int k = 0; k < kPlanKept; ++k)
        if (k * kPlanRound < rows) place(kept[k], k * kPlanRound + tid * 4, round++);
    for (int r0 = kPlanKept * kPlanRound; r0 < rows; r0 += kPlanRound) place(buckets(r0 + tid * 4), r0 + tid * 4, round++);
}

// ---- the slots' weighted sum, in slot order and fp32; slots of no expert take no part.  Four columns to a thread
template <typename TY>
__global__ __launch_bounds__(256) void moe_combine_kernel(const float* stage, const int32_t* ids, const float* weights, int T, int top_k,
                                                          int experts, int width, void* y, int ldy) {
    asm volatile("" ::: "v63");                          // a whole share of the register file (see quik_gemm.hip)
    const int per_row = (width + 3) / 4;
    const size_t at = ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
    if (at >= (size_t)T * per_row) return;
    const size_t t = at / per_row;
    const int n = (int)(at % per_row) * 4, count = min(4, width - n);
    const bool wide = width % 4 == 0;
    float v[4] = {};
    for (int j = 0; j < top_k; ++j) {
        const size_t r = t * top_k + j;
        const int e = ids[r];
        if (e < 0 || e >= experts) continue;
        const float w = weights[r];
        const float* const from = stage + r * width + n;
        float f[4] = {};
        if (wide) { const float4 u = *reinterpret_cast<const float4*>(from); f[0] = u.x; f[1] = u.y; f[2] = u.z; f[3] = u.w; }
        else for (int q = 0; q < count; ++q) f[q] = from[q];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = __builtin_fmaf(w, f[q], v[q]);
    }
    uint16_t* const to = static_cast<uint16_t*>(y) + t * ldy + n;
    if (count == 4 && ldy % 4 == 0 && (reinterpret_cast<uintptr_t>(y) & 7) == 0)
        *reinterpret_cast<uint2*>(to) = make_uint2(TY::round(v[0]) | (uint32_t)TY::round(v[1]) << 16, TY::round(v[2]) | (uint32_t)TY::round(v[3]) << 16);
    else
        for (int q = 0; q < count; ++q) to[q] = TY::round(v[q]);
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
    // (a grid's x dimension takes less than 2^32 threads)
    const size_t blocks = ((size_t)T * ((width + 3) / 4) + 255) / 256, slices = (blocks - 1) / (1 << 23) + 1;
    const dim3 grid((unsigned)((blocks - 1) / slices + 1), (unsigned)slices), threads(256);
    if (bf16) hipLaunchKernelGGL(moe_combine_kernel<Bf16>, grid, threads, 0, stream, stage, ids, weights, T, top_k, experts, width, y, ldy);
    else hipLaunchKernelGGL(moe_combine_kernel<Half>, grid, threads, 0, stream, stage, ids, weights, T, top_k, experts, width, y, ldy);
    return hipGetLastError();
}

}  // namespace quik
