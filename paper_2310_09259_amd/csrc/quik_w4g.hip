// Products with 4-bit weights in groups (layout: quik_w4g_device.h): y[t, n] = sum_k x[t, k] s[n, k / g] (q[n, k] -
// z[n, k / g]), for a dense layer and for the experts that a router chose.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "quik_gemm_device.h"
#include "quik_kernels.h"
#include "quik_w4g.h"
#include "quik_w4g_rows_device.h"

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
    const int tile = blockIdx.z * gridDim.x + blockIdx.x, b = tile / a.kt, kt = tile % a.kt;
    if (tile >= tiles) return;
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

// ---- few rows: the waves of a workgroup split K
//
// What bounds it: up to some 32 rows the weights, read once; beyond that the activations, which every workgroup reads whole
// out of L2.  A wave copies its tiles of 128 columns global -> LDS into a private ring of NST stages (no barrier until the
// waves add up), weights with the hint that they are read once: whole tiles of 1 KB, the row blocks' activations in
// pieces of 256 bytes a row, a channel block's scales and zero points in one copy.  (Activations loaded straight into
// registers as the matrix instructions want them, neighbouring lanes in different rows, take a clock of the CU's address
// path per lane: 64 x 16384 x 11008 came to 72 us that way, whatever the blocks.)
// A group's sum of x (q - z) is exact in its operands (16-bit activations, integers of at most eight bits) and held in
// fp32, and the scale is applied to it in fp32.  fp16 subtracts offset and zero point from the codes before the product;
// bf16, which has no packed subtraction, multiplies the codes with their offset of 128 and takes 136 + z times the sum
// of x off afterwards (an operand of ones gives it in the layout of the accumulators).
// Waves add up through LDS in wave order.
//
// MB, CB: row blocks and channel blocks of 16; NW waves.
// Rows of a block: consecutive ones (dense), or one (experts: a row at a time).  TOKEN: with weights a workgroup takes a
// token: the columns of its slots follow each other as if they were one long row, each slot's scales multiplied by its
// weight.
template <typename TY, int KG, int MB, int CB, int NW, int NST, bool TOKEN>
// (the bound, of more threads than a launch has, keeps the compiler to 256 registers where LDS would allow it more)
__global__ __launch_bounds__(512) void w4g_rows_kernel(W4gArgs a, int groups_n) {
    constexpr int PER = kCols / KG;
    constexpr bool SUMS = TY::kOffset < 1000.0f;
    constexpr int X_BYTES = MB * 16 * 256, S_AT = X_BYTES + CB * kTileBytes, STAGE = S_AT + CB * 256;
    constexpr int X_COPIES = MB * 4, LPS = X_COPIES + 2 * CB;
    static_assert((NST - 1) * LPS < 64, "vmcnt range");
    constexpr int RING = NW * NST * STAGE, RED = NW * MB * CB * 1024;
    if constexpr (MB * CB > 2) asm volatile("" ::: "v255");   // a whole share of the register file (see quik_gemm.hip)
    else asm volatile("" ::: "v127");
    __shared__ __align__(1024) uint8_t lds[RING > RED ? RING : RED];     // rings; then the partial sums
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
    const int id = gemm_dev::xcd_contiguous_id(blockIdx.x, gridDim.x);
    const int b0 = id % groups_n * CB, block = id / groups_n;

    RowSource src{0, block * MB * 16, min(MB * 16, a.rows - block * MB * 16), false};
    if (TOKEN) {
        src = RowSource{0, block, 1, false};
    } else if (a.ids) {
        const int e = a.ids[block];
        src = RowSource{e >= 0 && e < a.experts ? e : -1, block, 1, false};
    }
    // ---- where this lane's copies come from.  x: by offsets from the first row; copy i brings rows
    // 4 i .. 4 i + 3, its piece p of a row into place p ^ (row % 16), and zeros beyond the rows or beyond K
    const uint8_t* xbase = static_cast<const uint8_t*>(a.x);
    if (!a.ids) xbase += (size_t)src.first * a.ldx * 2;
    else xbase += (size_t)(TOKEN ? (a.x_per_slot ? block * a.top_k : block)
                                 : (a.x_per_slot ? block : block / a.top_k)) * a.ldx * 2;
    const gemm_dev::v4i rx = whole_rsrc(xbase);
    uint32_t vo[X_COPIES];
#pragma unroll
    for (int i = 0; i < X_COPIES; ++i) {
        const int r = 4 * i + g;
        vo[i] = r < src.count ? (uint32_t)r * (uint32_t)(a.ldx * 2) + ((l16 ^ (r & 15)) << 4) : kBeyond;
    }
    // a block's scales in the first 128 bytes of its 256, its zero points (or zeros) in the second
    const size_t tile0 = (size_t)b0 * a.w.kt;
    const bool is_scale = lane < 8 * PER, is_zero = a.w.zeros && lane >= 32 && lane < 32 + 4 * PER;
    const uint32_t per_tile = is_zero ? kBlock * PER : kBlock * PER * 2;

    // TOKEN: lane j has slot j's expert and weight (read from memory tile by tile, they would hold up every copy)
    const int slot_r = block * a.top_k + min(lane, a.top_k - 1);
    const int slot_e = TOKEN ? a.ids[slot_r] : 0;
    const float slot_w = TOKEN ? a.weights[slot_r] : 0.0f;

    uint8_t* const ring = lds + wave * (NST * STAGE);
    const uint32_t ring_addr = gemm_dev::lds_addr(ring);
    const int tiles = src.expert < 0 ? 0 : TOKEN ? a.top_k * a.w.kt : a.w.kt;
    const int first = tiles * wave / NW, last = tiles * (wave + 1) / NW;
    // The next tile of this wave's range, or past its end the last one again -> the weight of its slot.  (next_kt, next_j: its
    // columns and its slot; a division per tile would take longer than the tile)
    int next = first, next_j = TOKEN && tiles > 0 ? first / a.w.kt : 0, next_kt = first - next_j * a.w.kt;
    auto issue = [&](int slot) {
        const int kt = next_kt;
        int e = src.expert, room = a.w.K;
        uint32_t at = 0;
        float weight = 1.0f;
        if constexpr (TOKEN) {
            e = __builtin_amdgcn_readlane(slot_e, next_j);
            const bool on = e >= 0 && e < a.experts;
            e = on ? e : 0;
            const float v = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, slot_w), next_j));
            weight = on ? v : 0.0f;
            room = on ? room : 0;
            at = (uint32_t)(a.x_per_slot ? next_j : 0) * (uint32_t)(a.ldx * 2);
        }
        if (next + 1 < last) {
            ++next;
            ++next_kt;
            if (TOKEN && next_kt == a.w.kt) { next_kt = 0; ++next_j; }
        }
        room -= kt * kCols;
        at += (uint32_t)kt * 256;
        const uint32_t dst = ring_addr + slot * STAGE;
        const gemm_dev::v4i rw = whole_rsrc(a.w.codes + e * a.w.codes_e + tile0 * kTileBytes);
        const uint8_t* const s0 = a.w.scales + e * a.w.scales_e + tile0 * (kBlock * PER * 2);
        const gemm_dev::v4i rs = whole_rsrc(s0);
        const uint32_t zeros_at = a.w.zeros ? (uint32_t)(a.w.zeros + e * a.w.zeros_e + tile0 * (kBlock * PER) - s0) : 0u;
        const uint32_t so = is_zero ? zeros_at + (lane - 32) * 4 : lane * 4;
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            const uint32_t tile = (uint32_t)min(c, a.w.nt - 1 - b0) * a.w.kt + kt;
            gemm_dev::dma16_once(rw, dst + X_BYTES + c * kTileBytes, lane * 16 + tile * kTileBytes);
            gemm_dev::dma4(rs, dst + S_AT + c * 256, is_scale || is_zero ? so + tile * per_tile : kBeyond);
        }
#pragma unroll
        for (int i = 0; i < X_COPIES; ++i)
            gemm_dev::dma16(rx, dst + i * 1024, (l16 ^ ((4 * i + g) & 15)) * 8 < room ? vo[i] : kBeyond, at);
        return weight;
    };

    v4f acc[MB][CB] = {};
    const v4u ones = v4u{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    uint32_t mask = 0x000F000Fu, bits = TY::kBits;       // (in registers: two literals would cost an instruction more)
    asm volatile("" : "+s"(mask), "+v"(bits));
    auto multiply = [&](const uint8_t* st, float weight) {
        v4u w[CB];
#pragma unroll
        for (int c = 0; c < CB; ++c) w[c] = *reinterpret_cast<const v4u*>(st + X_BYTES + c * kTileBytes + lane * 16);
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            v4f part[MB][CB] = {}, sum[MB] = {};
            int zero[CB];
            float scale[CB];
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                const uint8_t* const sz = st + S_AT + c * 256 + l16 * PER + p;
                scale[c] = (float)*reinterpret_cast<const _Float16*>(st + S_AT + c * 256 + (l16 * PER + p) * 2);
                if constexpr (TOKEN) scale[c] *= weight;
                zero[c] = (int)(8.0f + TY::kOffset) + *reinterpret_cast<const int8_t*>(sz + 128);
            }
#pragma unroll
            for (int s = p * (4 / PER); s < (p + 1) * (4 / PER); ++s) {
                v4u x[MB];
#pragma unroll
                for (int m = 0; m < MB; ++m)
                    x[m] = *reinterpret_cast<const v4u*>(st + (m * 16 + l16) * 256 + (((s * 4 + g) ^ l16) << 4));
                if constexpr (SUMS) {
#pragma unroll
                    for (int m = 0; m < MB; ++m) sum[m] = TY::mfma(x[m], ones, sum[m]);
                }
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    const _Float16 z1 = (_Float16)(short)zero[c];
                    const v2h z2 = v2h{z1, z1};
                    v4u b;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t u = ((w[c][s] >> (4 * i)) & mask) | bits;
                        b[i] = SUMS ? u : __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, u) - z2);
                    }
#pragma unroll
                    for (int m = 0; m < MB; ++m) part[m][c] = TY::mfma(x[m], b, part[m][c]);
                }
            }
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int c = 0; c < CB; ++c)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v = part[m][c][r];
                        if constexpr (SUMS) v = __builtin_fmaf(-(float)zero[c], sum[m][r], v);
                        acc[m][c][r] = __builtin_fmaf(scale[c], v, acc[m][c][r]);
                    }
        }
    };

    if (first < last) {
        float ahead[NST - 1];                            // the weights of the tiles under way
#pragma unroll
        for (int d = 0; d < NST - 1; ++d) ahead[d] = issue(d);
        int slot = 0, fill = NST - 1;
        for (int vt = first; vt < last; ++vt) {
            __builtin_amdgcn_s_waitcnt(0xC07F);          // lgkmcnt(0): the reads of the stage about to be filled are done
            const float weight = issue(fill);
            gemm_dev::wait_vm<(NST - 1) * LPS>();        // tile vt has landed (this wave's own copies)
            asm volatile("" ::: "memory");
            multiply(ring + slot * STAGE, ahead[0]);
#pragma unroll
            for (int d = 0; d < NST - 2; ++d) ahead[d] = ahead[d + 1];
            ahead[NST - 2] = weight;
            slot = slot + 1 == NST ? 0 : slot + 1;
            fill = fill + 1 == NST ? 0 : fill + 1;
        }
        gemm_dev::wait_vm<0>();
    }
    __syncthreads();                                     // every ring is dead
    float4 (*red)[MB * CB][64] = reinterpret_cast<float4 (*)[MB * CB][64]>(lds);
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int c = 0; c < CB; ++c) red[wave][m * CB + c][lane] = make_float4(acc[m][c][0], acc[m][c][1], acc[m][c][2], acc[m][c][3]);
    __syncthreads();

    // ---- the sums in wave order: a wave finishes a block, or both halves of a pair, and then the next
    const int step = a.glu ? 2 : 1;
    for (int q = wave * step; q < MB * CB; q += NW * step) {
        const int m = q / CB, c = q % CB;
        const int n = (a.glu ? (b0 + c) >> 1 : b0 + c) * kBlock + l16;
        if (n >= a.width || m * 16 >= src.count) continue;
        float v[2][4] = {};
        for (int h = 0; h < step; ++h) {
            for (int w = 0; w < NW; ++w) {
                const float4 f = red[w][q + h][lane];
                v[h][0] += f.x; v[h][1] += f.y; v[h][2] += f.z; v[h][3] += f.w;
            }
            if (a.bias) {
                float bias = 0.0f;
                if (TOKEN) {
                    for (int j = 0; j < a.top_k; ++j) {
                        const int e = a.ids[block * a.top_k + j];
                        if (e >= 0 && e < a.experts) bias = __builtin_fmaf(a.weights[block * a.top_k + j], TY::load(a.bias, (size_t)e * a.w.N + n), bias);
                    }
                } else if (src.expert >= 0) {
                    bias = TY::load(a.bias, (size_t)src.expert * a.w.N + n + h * a.width);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) v[h][r] += bias;
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = m * 16 + 4 * g + r;
            if (i >= src.count) continue;
            const float y = src.expert < 0 ? 0.0f : a.glu ? silu_product(v[0][r], v[1][r]) : v[0][r];
            const size_t row = (size_t)src.first + i;
            if (a.weights && !TOKEN) a.stage[row * a.width + n] = y;
            else static_cast<uint16_t*>(a.y)[row * a.ldy + n] = TY::round(y);
        }
    }
}

template <typename TY, int KG, int MB, int CB, int NW, int NST>
hipError_t launch_rows(const W4gArgs& a, hipStream_t stream) {
    const int groups_n = (a.w.nt + CB - 1) / CB;
    const dim3 threads(NW * 64);
    if constexpr (MB == 1) {
        if (a.weights && !a.glu) {
            hipLaunchKernelGGL((w4g_rows_kernel<TY, KG, 1, CB, NW, NST, true>), dim3((unsigned)(a.rows / a.top_k) * groups_n), threads, 0, stream, a, groups_n);
            return hipGetLastError();
        }
    }
    int blocks = (a.rows + MB * 16 - 1) / (MB * 16);
    if (a.ids) blocks = a.rows;
    hipLaunchKernelGGL((w4g_rows_kernel<TY, KG, MB, CB, NW, NST, false>), dim3((unsigned)blocks * groups_n), threads, 0, stream, a, groups_n);
    return hipGetLastError();
}

template <typename TY, int KG>
hipError_t rows_dispatch(const W4gArgs& a, int form, hipStream_t stream) {
    switch (form) {
        case kW4gRows16x16: return launch_rows<TY, KG, 1, 1, 8, 3>(a, stream);
        case kW4gRows16x32Wide: return launch_rows<TY, KG, 1, 2, 8, 2>(a, stream);
        case kW4gRows16x32: return launch_rows<TY, KG, 1, 2, 4, 2>(a, stream);
        case kW4gRows16x64: return launch_rows<TY, KG, 1, 4, 4, 2>(a, stream);
        case kW4gRows32x32: return launch_rows<TY, KG, 2, 2, 6, 2>(a, stream);
        case kW4gRows32x64: return launch_rows<TY, KG, 2, 4, 6, 2>(a, stream);
        default: return hipErrorInvalidValue;
    }
}

hipError_t launch_w4g_rows(const W4gArgs& a, int form, hipStream_t stream) {
    switch (a.group + a.bf16) {
        case 32: return rows_dispatch<Half, 32>(a, form, stream);
        case 64: return rows_dispatch<Half, 64>(a, form, stream);
        case 128: return rows_dispatch<Half, 128>(a, form, stream);
        case 33: return rows_dispatch<Bf16, 32>(a, form, stream);
        case 65: return rows_dispatch<Bf16, 64>(a, form, stream);
        case 129: return rows_dispatch<Bf16, 128>(a, form, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_weight_pack_w4g(const void* w_q, int ldw, const void* w_scale, const void* w_zero, int N, int K, int group,
                                  int glu, int experts, void* w4, hipStream_t stream) {
    const Layout l = layout(N, K, group, w_zero != nullptr, glu != 0, experts);
    uint8_t* const base = static_cast<uint8_t*>(w4);
    PackArgs a{static_cast<const uint8_t*>(w_q), ldw, static_cast<const uint16_t*>(w_scale), static_cast<const int8_t*>(w_zero),
               N, K, group ? (K - 1) / group + 1 : 1, group ? group : K, l.kg, glu, l.nt, l.kt,   // (a group may be near 2^31)
               reinterpret_cast<uint32_t*>(base), reinterpret_cast<uint16_t*>(base + l.scales_at),
               reinterpret_cast<int8_t*>(base + l.zeros_at)};
    // up to 2^16 x 2^8 tiles of 256 threads: more than a grid's x takes
    const int tiles = l.nt * l.kt, slices = (tiles - 1) / (1 << 23) + 1;
    hipLaunchKernelGGL(pack_w4g_kernel, dim3((tiles - 1) / slices + 1, experts, slices), dim3(256), 0, stream, a);
    return hipGetLastError();
}

namespace { std::atomic<int> g_form{-1}; }
void set_w4g_form(int form) { g_form.store(form, std::memory_order_relaxed); }

// Up to 16 rows, and for a row (or token) of experts at a time, the choice goes by the channel blocks of all of them together
// (us, weights from HBM, K = 4096 unless noted):
//  - one block per CU or fewer: single blocks and eight waves (N = 4096, 1 row: 6.0 against 6.7 with pairs, 7.4 with four
//    waves); paired halves, and up to two per CU: pairs and eight waves;
//  - more: pairs and four waves, two and three workgroups to a CU (N = 15360, K = 5120: 11.4 against 13.8 with eight waves);
//    from six blocks per CU on four of them at a time (N = 28672, K = 8192: 24.9 against 26.9).
// More rows of a dense layer: the least of an estimate, rounds of workgroups, one to a CU, times the tiles of 128 columns
// that a wave (or group of waves) goes through, times what such a step takes, plus a start.  Measured steps: 1.3 us and 1.75
// for 32 x 32 and 32 x 64 (six waves split K), 0.95 and 1.4 for tiles of 32 x 128 and 64 x 128 (two groups split K), 1.2,
// 1.95 and 3.3 for 128 x 128, 256 x 128 and 256 x 256, in fp16 with groups of 128; small groups and bf16 make them up to a half
// longer, by about the same factor in all.  (256 x 256 has come to 3.6; over 390 sizes from 24 to 4096 rows, both types, groups of
// 32, 64 and 128, the choice takes 0.2 % longer than the best of these kernels and at most 7 %, with 3.6 up to 13 %.)  N = 11008, chosen : best other one: 24 rows 14.3 : 17.4, 48 rows
// 19.1 : 23.7, 128 rows 24.7 : 34, 256 rows 41.7 : 47.8, 512 rows 62 : 73, 1024 rows 113 : 126, 2048 rows 199 : 232; N = 4096,
// 1024 rows 44.5 : 49.4; N = 28672, K = 8192, 4096 rows 1660 : 1870.
// Experts by a plan: workgroups of four waves, several to a CU, since each has few steps, and its start (its rows, its
// first tiles) and its end would leave the CU idle.  Tiles of 32 rows up to about a hundred rows to an expert, then of 64 (in
// brackets the best with one workgroup to a CU): 64 experts of 2048 x 2816 in halves, bf16, groups of 64, 28 rows each 103 : 122 (150);
// fp16, 256 rows each 345 : 295 (424); of 1408 x 2048, summed up, 256 rows each 232 : 205 (288); eight of 4096 x 4096 in
// halves, 16 rows each 39.3 : 44 (42), 128 rows each 84 : 85 (105), 512 rows each 241 : 196 (256).
// tile256: whether there is a 256 x 256 tile for the layer (dense, no paired halves, stored groups of 128)
static int choose_w4g_form(int rows, int blocks, int kt, bool glu, int experts, bool by_rows, bool tile256, int cus) {
    if (by_rows || (!experts && rows <= 16)) {
        const double all = (double)blocks * (by_rows ? rows : 1);
        if (all <= cus && !glu) return kW4gRows16x16;
        if (all <= 2 * cus) return kW4gRows16x32Wide;
        return all >= 6 * cus ? kW4gRows16x64 : kW4gRows16x32;
    }
    if (experts) return rows <= 100.0 * experts ? kW4gTile32x128Small : kW4gTile64x128Small;
    struct Cost { int form, rows, blocks, k_split; double start, step; };
    static const Cost costs[] = {
        {kW4gRows32x32, 32, 2, 6, 5.0, 1.3},     {kW4gRows32x64, 32, 4, 6, 5.0, 1.75},    {kW4gTile32x128, 32, 8, 2, 3.0, 0.95},
        {kW4gTile64x128, 64, 8, 2, 3.0, 1.4},    {kW4gTile128x128, 128, 8, 1, 3.0, 1.2},  {kW4gTile256x128, 256, 8, 1, 3.0, 1.95},
        {kW4gTile256x256, 256, 16, 1, 3.0, 3.3},
    };
    int best = kW4gTile256x128;
    double least = 1e30;
    for (const Cost& c : costs) {
        if (!tile256 && c.form == kW4gTile256x256) continue;
        const double tiles = (double)((rows + c.rows - 1) / c.rows) * ((blocks + c.blocks - 1) / c.blocks);
        const double t = c.start + ceil(tiles / cus) * ((kt + c.k_split - 1) / c.k_split) * c.step;
        if (t < least) { least = t; best = c.form; }
    }
    return best;
}

W4gChoice resolve_w4g(int rows, int top_k, bool combine, int blocks, int kt, int group, bool glu, int experts, int cus) {
    // a row (or a token and its slots) at a time where hardly two rows share an expert: no plan, no sums in memory
    W4gChoice c;
    c.by_rows = experts && rows <= experts;
    c.by_token = c.by_rows && combine && !glu;
    const bool tile256 = !glu && !experts && group == 128;
    c.form = g_form.load(std::memory_order_relaxed);
    if (c.form < 0) c.form = choose_w4g_form(c.by_token ? rows / top_k : rows, blocks, kt, glu, experts, c.by_rows, tile256, cus);
    // (a form that was set may not be one for this product)
    if (c.by_rows && c.form > kW4gRows16x64) c.form = kW4gRows16x32;
    if (experts && !c.by_rows && c.form < kW4gTile32x128) c.form = kW4gTile32x128Small;
    if (glu && c.form == kW4gRows16x16) c.form = kW4gRows16x32Wide;
    if (!tile256 && c.form == kW4gTile256x256) c.form = kW4gTile256x128;
    return c;
}

// (what a grid's x dimension takes is counted in threads)
static bool fits_a_grid(const W4gArgs& a, const W4gChoice& c) {
    static const struct { int rows, blocks, threads; } tile[kW4gForms] = {
        {16, 1, 512}, {16, 2, 512}, {16, 2, 256}, {16, 4, 256}, {32, 2, 384}, {32, 4, 384},
        {32, 8, 512}, {64, 8, 512}, {128, 8, 512}, {256, 8, 512}, {256, 16, 512}, {32, 8, 256}, {64, 8, 256}};
    const auto& t = tile[c.form];
    const size_t groups = (a.w.nt + t.blocks - 1) / t.blocks;
    const size_t rows = c.by_token ? a.rows / a.top_k : c.by_rows ? a.rows
                        : a.ids ? a.rows / t.rows + min(a.rows, a.experts + 1) : (a.rows + t.rows - 1) / t.rows;
    return rows * groups * t.threads <= 0xFFFFFFFFu;
}

hipError_t launch_w4g(const W4gArgs& args, hipStream_t stream) {
    W4gArgs a = args;
    const int cus = compute_units();
    const W4gChoice c = resolve_w4g(a.rows, a.top_k, a.weights != nullptr, a.w.nt, a.w.kt, a.group, a.glu, a.ids ? a.experts : 0, cus > 0 ? cus : 256);
    if (!fits_a_grid(a, c)) return hipErrorInvalidConfiguration;
    if (c.by_rows) a.plan = nullptr;
    else if (a.ids) {
        if (hipError_t rc = launch_moe_plan(a.ids, a.rows, a.experts, a.plan, stream); rc != hipSuccess) return rc;
    }
    const hipError_t rc = c.form < kW4gTile32x128 ? launch_w4g_rows(a, c.form, stream) : launch_w4g_tiles(a, c.form, stream);
    if (rc != hipSuccess || !a.weights || c.by_token) return rc;
    return launch_moe_combine(a.stage, a.ids, a.weights, a.rows / a.top_k, a.top_k, a.experts, a.width, a.bf16, a.y, a.ldy, stream);
}

}  // namespace quik
