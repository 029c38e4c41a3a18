// Products with 4-bit weights in groups for many rows (quik_w4g.hip has the few): tiles of the output on the 16-bit
// matrix instructions.
//
// What bounds it: the matrix pipes and, in turn rather than at the same time (a step's clocks come close to the sum of both), the
// vector instructions that widen the weights.  A wave of IB x JB blocks of 16 x 16 outputs reads its weights from LDS in the
// lane order that the layout gives them and widens them for all its IB row blocks: eight weights take 11 to 19 vector
// instructions of 4 clocks, against IB / 4 matrix instructions of 16.  128 rows to a wave keep that at a third to a half of the
// matrix time; fewer rows cannot.  Widened weights in LDS, once per workgroup, would be read back at 1.5 times the bytes
// that the activations already take of it.
//
// The widened weights are the integers q - z, exact in either type, and the scales are applied in fp32: nothing is rounded to 16
// bits but the output.
//   FOLD   a group's sums of products have registers of their own, and are added up with one fused multiply-add per output and
//          group.
//   else   (256 x 256, which has no room for that; groups of 128) the sums are in units of their channel's scale.  Where the next
//          group begins they are multiplied by the quotient of the old scale and the new one, two roundings of 2^-24, and the
//          units come off at the end.  A k-step goes through the channel blocks pair by pair, with all its row blocks in
//          registers: the weights widened ahead are those of a pair, not of all blocks.
// For 4096 x 8192 x 28672 in fp16 : bf16, groups of 128, 256 x 256 takes 1660 : 1790 us and 256 x 128 1880 : 2000.
//
// The activations of 128 columns go through LDS, two stages, copied without passing through registers; rows are 256
// bytes, their sixteen 16-byte pieces exchanged by the row's number so that sixteen rows' pieces of one k fall into
// distinct banks.  Columns beyond K are zeros there (copies out of range), so that weights beyond K may be anything finite.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "quik_gemm_device.h"
#include "quik_w4g.h"
#include "quik_w4g_rows_device.h"

namespace quik {

namespace {

using namespace w4g;
using gemm_dev::v4i;

// The eight weights of one dword as integers q - z, exact in either type, in eight pieces of work (`part`, 0 .. 7) that stand
// between matrix instructions; `zero` is z + 8.  fp16: (1024 + u) - (1032 + z)
struct HalfCodes {
    v2h zero;
    __device__ __forceinline__ void set(int z8) {
        const _Float16 c = (_Float16)(float)(1024 + z8);
        zero = v2h{c, c};
    }
    __device__ __forceinline__ void widen(int part, uint32_t w, v4u& b, uint32_t mask, uint32_t bits, float) const {
        const int i = part >> 1;
        if (part & 1) return;
        b[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, ((w >> (4 * i)) & mask) | bits) - zero);
    }
};
// bf16: (1024 + u) - (1032 + z) in fp32, as one fused multiply-add that takes the fp16 half (by a 1 that the compiler does not
// see, or it makes a conversion and an addition of it)
struct Bf16Codes {
    float zero;
    __device__ __forceinline__ void set(int z8) { zero = -(float)(1024 + z8); }
    __device__ __forceinline__ void widen(int part, uint32_t w, v4u& b, uint32_t mask, uint32_t bits, float one) const {
        typedef __bf16 v2b __attribute__((ext_vector_type(2)));
        const int i = part >> 1;
        if (part & 1) {
            const v2h u = __builtin_bit_cast(v2h, (uint32_t)b[i]);
            const v2b v = {(__bf16)__builtin_fmaf((float)u[0], one, zero), (__bf16)__builtin_fmaf((float)u[1], one, zero)};
            b[i] = __builtin_bit_cast(uint32_t, v);
        } else {
            b[i] = ((w >> (4 * i)) & mask) | bits;
        }
    }
};
template <typename TY> struct CodesOf { typedef HalfCodes type; };
template <> struct CodesOf<Bf16> { typedef Bf16Codes type; };

// IB x JB blocks of 16 to a wave, WM x WN waves to a tile, KS groups of such waves that take every KS-th stage each and add
// up through LDS at the end, in their order.  NST stages to a group: two where a stage is long enough to hide the next
// one's way from memory (256 x 256: 3.7 us), three or four for the small tiles.  OCC waves per SIMD: two; four for the
// smallest tile of experts, whose workgroups' starts and ends go on behind each other's products.
template <typename TY, int KG, int IB, int JB, int WM, int WN, int KS, int NST, int OCC, bool FOLD>
__global__ __launch_bounds__(OCC == 2 ? 512 : WM * WN * KS * 64, OCC) void w4g_tiles_kernel(W4gArgs a, int tiles_m) {
    constexpr int NW = WM * WN, BM = IB * WM * 16, BB = JB * WN, PER = kCols / KG;
    constexpr int COPIES = BM / 4 / NW;                  // of four rows each, per wave and stage
    static_assert(FOLD || (PER == 1 && KS == 1 && NST == 2 && IB == 8 && JB == 4), "a group to a stage; two pairs of channel blocks, eight pieces of a block each");
    static_assert(BM % (4 * NW) == 0 && BB % NW == 0 && JB % 2 == 0 && JB <= IB, "whole copies, whole pairs, at most a block widened per row block");
    // the whole share of the register file (see quik_gemm.hip); of the 168 registers of three waves all but the last
    if constexpr (OCC == 2) asm volatile("" ::: "v255");
    else if constexpr (OCC == 3) asm volatile("" ::: "v166");
    else asm volatile("" ::: "v127");
    constexpr int W_COPIES = BB / NW;                    // of one weight tile each, per wave and stage
    // scales and zero points: with two stages straight into registers, a stage ahead; through LDS, BPC blocks to a copy of 256
    // bytes, with more stages, where the wait for them must not be one for later stages, and where small groups' scales would
    // fill the registers (256 x 128 in groups of 32, 2048 x 4096 x 11008: 250 us, 320 with some in scratch memory)
    constexpr bool S_LDS = NST > 2 || (FOLD && PER > 1 && IB == 8) || (PER == 4 && OCC == 4);
    constexpr int BPC = 4 / PER, S_COPIES = !S_LDS ? 0 : BB / BPC > NW ? BB / BPC / NW : 1;
    constexpr int X_BYTES = BM * 256, S_AT = X_BYTES + BB * kTileBytes, STAGE = S_AT + NW * S_COPIES * 256;
    __shared__ __align__(1024) uint8_t all_lds[KS * NST * STAGE];
    static_assert(KS == 1 || KS * NST * STAGE >= (KS - 1) * NW * IB * JB * 1024, "the groups' sums fit the rings");

    const int tid = threadIdx.x, lane = tid & 63, all = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = all / NW, wave = all % NW;            // K group, wave in it
    const int l16 = lane & 15, g = lane >> 4, wm = wave / WN, wn = wave % WN;
    uint8_t* const lds = all_lds + kg * (NST * STAGE);

    // eight row tiles at a time are swept along the channels, the row tiles next to each other
    const int tiles_n = (a.w.nt + BB - 1) / BB;
    const int id = gemm_dev::xcd_contiguous_id(blockIdx.x, gridDim.x);
    constexpr int GM = 8;
    const int grp = id / (GM * tiles_n), rem = id % (GM * tiles_n), gsz = min(GM, tiles_m - grp * GM);
    const int tile_m = grp * GM + rem % gsz, b0 = rem / gsz * BB;

    RowSource src{0, tile_m * BM, min(BM, a.rows - tile_m * BM), false};
    if (a.ids) {
        src = planned_rows(a.plan, a.experts, tile_m, BM);
        if (src.count == 0) return;
    }
    const int32_t* const list = src.listed ? a.plan + a.experts + 2 + src.first : nullptr;
    const int kt_end = src.expert >= 0 ? (a.w.kt + KS - 1) / KS : 0;     // stages of every group
    const size_t e = src.expert > 0 ? src.expert : 0;

    // ---- where this lane's copies come from: row 4 (copy * NW + wave) + lane / 16, piece (lane % 16) ^ (row % 16)
    const uint8_t* xbase = static_cast<const uint8_t*>(a.x);
    if (!list) xbase += (size_t)src.first * a.ldx * 2;
    const v4i rx = whole_rsrc(xbase);
    uint32_t vo[FOLD ? COPIES : 1];                      // not FOLD: of copy 0, the others lie 4 NW rows apart each
#pragma unroll
    for (int c = 0; c < (FOLD ? COPIES : 1); ++c) {
        const int r = 4 * (c * NW + wave) + (lane >> 4), in = FOLD ? min(r, src.count - 1) : r;
        uint32_t row = in;
        if (list) {
            row = list[in];
            if (!a.x_per_slot) row /= (uint32_t)a.top_k;
        }
        vo[c] = row * (uint32_t)(a.ldx * 2) + (((lane & 15) ^ (r & 15)) << 4);
    }
    // copy c of this group's stage kt: the rows' activations, then the weight tiles.  (Beyond the end: zeros, and the last
    // weights again; a branch would cut the loop's schedule)
    const uint8_t* const codes = a.w.codes + e * a.w.codes_e;
    const v4i rw = whole_rsrc(codes + (size_t)b0 * a.w.kt * kTileBytes);
    const uint32_t lds0 = gemm_dev::lds_addr(lds) + wave * 1024;
    const uint8_t* const s0 = a.w.scales + e * a.w.scales_e + (size_t)b0 * a.w.kt * (kBlock * PER * 2);
    const v4i rs = whole_rsrc(s0);
    const uint32_t zeros_at = a.w.zeros ? (uint32_t)(a.w.zeros + e * a.w.zeros_e + (size_t)b0 * a.w.kt * (kBlock * PER) - s0) : 0u;
    auto copy = [&](int kt, int c, uint32_t slot) {      // (slot: its bytes in the ring)
        const uint32_t dst = lds0 + slot;
        const int tile_k = kt * KS + kg, from = min(tile_k, a.w.kt - 1);
        if (c < COPIES) {
            const int r = 4 * (c * NW + wave) + (lane >> 4), k = ((lane & 15) ^ (r & 15)) << 3;
            if constexpr (FOLD)
                gemm_dev::dma16(rx, dst + c * NW * 1024, k < a.w.K - tile_k * kCols ? vo[c < COPIES ? c : 0] + (uint32_t)tile_k * 256 : kBeyond, 0);
            else                                         // (rows beyond the last: zeros)
                gemm_dev::dma16(rx, dst + c * NW * 1024, ((k < a.w.K - tile_k * kCols) & (r < src.count)) ? vo[0] : kBeyond,
                                (uint32_t)(c * NW * 4) * (uint32_t)(a.ldx * 2) + (uint32_t)tile_k * 256);
        } else if (c >= COPIES + W_COPIES) {             // lane: dword `in` of block lane / (16 PER)'s 8 PER scales and 4 PER zero points
            const int copy_at = (c - COPIES - W_COPIES) * NW + wave, in = lane % (16 * PER);
            const int block = copy_at * BPC + lane / (16 * PER);
            const uint32_t tile = (uint32_t)min(block, a.w.nt - 1 - b0) * a.w.kt + from;
            const uint32_t vo_s = in < 8 * PER ? tile * (kBlock * PER * 2) + in * 4
                                  : in < 12 * PER && a.w.zeros ? zeros_at + tile * (kBlock * PER) + (in - 8 * PER) * 4 : kBeyond;
            gemm_dev::dma4(rs, dst + S_AT + (c - COPIES - W_COPIES) * NW * 256 - wave * 768, vo_s);
        } else {
            const int block = (c - COPIES) * NW + wave;
            const uint32_t tile = (uint32_t)min(block, a.w.nt - 1 - b0) * a.w.kt + from;
            gemm_dev::dma16(rw, dst + X_BYTES + (c - COPIES) * NW * 1024, lane * 16, tile * kTileBytes);
        }
    };

    // ---- the scales of this wave's channel blocks, through registers
    // (uniform addresses, 32-bit offsets of the lanes; without zero points the scales are read in their place, and masked)
    const uint8_t* const scales = a.w.scales + e * a.w.scales_e;
    const uint8_t* const zeros = a.w.zeros ? a.w.zeros + e * a.w.zeros_e : scales;
    const uint32_t zero_mask = a.w.zeros ? 0xFFFFFFFFu : 0u;
    // of this stage and the next: zero points, PER of channel l16; not FOLD: the scale in the low half, the zero point above it
    uint32_t sz[JB], scn[JB], zen[JB];
    // FOLD: the scales of channels 4 g .. 4 g + 3, whose sums this lane has, [4][PER]; of the next stage; of the last group
    uint32_t sf[JB][2 * PER] = {}, sfn[JB][2 * PER] = {};
    _Float16 sl[JB][4] = {};
    auto fetch = [&](int kt, int j) {
        if constexpr (!FOLD) {                           // (32-bit addresses)
            const uint32_t t = (uint32_t)min(wn * JB + j, a.w.nt - 1 - b0) * a.w.kt + (uint32_t)min(kt, a.w.kt - 1);
            const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(s0), 0, kRange, 0x00020000);
            scn[j] = __builtin_amdgcn_raw_buffer_load_b16(r, l16 * 2, t * (kBlock * 2), 0);
            zen[j] = __builtin_amdgcn_raw_buffer_load_b8(r, l16, zeros_at + t * kBlock, 0);
        } else {
            const size_t tile = (size_t)min(b0 + wn * JB + j, a.w.nt - 1) * a.w.kt + min(kt * KS + kg, a.w.kt - 1);
            const uint2* f = reinterpret_cast<const uint2*>(scales + tile * (kBlock * PER * 2) + (uint32_t)g * (8 * PER));
#pragma unroll
            for (int q = 0; q < PER; ++q) { const uint2 v = f[q]; sfn[j][2 * q] = v.x; sfn[j][2 * q + 1] = v.y; }
            const uint8_t* z = zeros + tile * (kBlock * PER) + (uint32_t)(l16 * PER);
            if constexpr (PER == 1) zen[j] = *z;
            else if constexpr (PER == 2) zen[j] = *reinterpret_cast<const uint16_t*>(z);
            else zen[j] = *reinterpret_cast<const uint32_t*>(z);
        }
    };
    auto take = [&](uint32_t slot) {
#pragma unroll
        for (int j = 0; j < JB; ++j) {
            if constexpr (S_LDS) {
                const uint8_t* const at = lds + slot + S_AT + (wn * JB + j) * (64 * PER) + 32 * PER + l16 * PER;
                if constexpr (PER == 1) sz[j] = *at;
                else if constexpr (PER == 2) sz[j] = *reinterpret_cast<const uint16_t*>(at);
                else sz[j] = *reinterpret_cast<const uint32_t*>(at);
            } else if constexpr (FOLD) {
                sz[j] = zen[j] & zero_mask;
            } else {
                sz[j] = scn[j] | (zen[j] & zero_mask) << 16;
            }
        }
    };
    // FOLD, at the start of a stage: its scales, and what the sums of the last group still need
    auto take_fold = [&](uint32_t slot) {
#pragma unroll
        for (int j = 0; j < JB; ++j) {
#pragma unroll
            for (int r = 0; r < 4; ++r) sl[j][r] = __builtin_bit_cast(_Float16, (uint16_t)(sf[j][(r * PER + PER - 1) / 2] >> (16 * ((r * PER + PER - 1) & 1))));
            if constexpr (S_LDS) {
                const uint2* f = reinterpret_cast<const uint2*>(lds + slot + S_AT + (wn * JB + j) * (64 * PER) + g * (8 * PER));
#pragma unroll
                for (int q = 0; q < PER; ++q) { const uint2 v = f[q]; sf[j][2 * q] = v.x; sf[j][2 * q + 1] = v.y; }
            } else {
#pragma unroll
                for (int q = 0; q < 2 * PER; ++q) sf[j][q] = sfn[j][q];
            }
        }
    };

    v4f acc[IB][JB] = {}, part[FOLD ? IB : 1][FOLD ? JB : 1] = {};
    // FOLD: row block i's sums of group p of this stage, -1: of the stage before
    auto fold = [&](int i, int p) {
#pragma unroll
        for (int j = 0; j < JB; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const _Float16 f = p < 0 ? sl[j][r] : __builtin_bit_cast(_Float16, (uint16_t)(sf[j][(r * PER + p) / 2] >> (16 * ((r * PER + p) & 1))));
                acc[i][j][r] = __builtin_fmaf((float)f, part[FOLD ? i : 0][FOLD ? j : 0][r], acc[i][j][r]);
            }
    };
    // FOLD: row blocks of the next units: a unit of two matrix instructions is over before a read of LDS returns, so they are
    // read seven units ahead, or three where the registers are full; weights of this k-step and the next.  (Not so far that the
    // next stage's are read before this stage's copies have all been issued, in its first two units: see READY.)  Else: the row
    // blocks of a k-step; weights of this pair of channel blocks and the next
    constexpr int PAIRS = JB / 2, UNITS = FOLD ? 4 * IB : 4 * PAIRS, COPIED = 2;
    constexpr int XR = !FOLD ? IB : IB * JB * 2 >= 32 || OCC > 2 ? 4 : 8, AHEAD = XR - 1 < UNITS - COPIED ? XR - 1 : UNITS - COPIED;
    constexpr int WB = FOLD ? JB : 2;                    // blocks whose weights are widened at a time
    v4u x[XR], b[2][WB];
    uint32_t w[WB];                                      // packed weights of the next k-step, or pair
    const int row_at = (wm * IB * 16 + l16) * 256, w_at = X_BYTES + wn * JB * kTileBytes + lane * 16;
    uint32_t cur = 0, nxt = STAGE, prv = (NST - 1) * STAGE;   // the ring's bytes of this, the next and the last stage
    // (not FOLD: from one address, the swizzle's by an exclusive or, so that there are not four of them to keep)
    static_assert(STAGE % 256 == 0, "the k-step is in the address's bits 6 and 7");
    const uint32_t row_of = gemm_dev::lds_addr(lds) + row_at + ((g ^ l16) << 4);
    auto row_block = [&](int i, int ks) {                // k-steps from 4 on are the next stage's
        if constexpr (!FOLD) {
            typedef __attribute__((address_space(3))) const v4u* lds_v4u;
            return *(lds_v4u)(uintptr_t)((((ks < 4 ? cur : nxt) + row_of) ^ ((ks & 3) << 6)) + i * (16 * 256));
        }
        return *reinterpret_cast<const v4u*>(lds + (ks < 4 ? cur : nxt) + row_at + i * (16 * 256) + ((((ks & 3) * 4 + g) ^ l16) << 4));
    };
    auto packed = [&](int j, int ks) {                   // block j's weights
        return *reinterpret_cast<const uint32_t*>(lds + (ks < 4 ? cur : nxt) + w_at + j * kTileBytes + (ks & 3) * 4);
    };
    uint32_t mask = 0x000F000Fu, bits = Half::kBits;     // (in registers: two literals would cost an instruction more)
    float one = 1.0f;
    asm volatile("" : "+s"(mask), "+v"(bits), "+s"(one));
    typename CodesOf<TY>::type s[JB];
    auto zero_of = [&](int j, int p) { return 8 + (int)(int8_t)(sz[j] >> (FOLD ? 8 * p : 16)); };
    // READY: before this unit of work a barrier says that the next stage is there, before the last one of all, FREE, another that
    // this stage is read and may be filled; the copies follow in the gaps of three units.  The wait at READY leaves the copies of
    // the NST - 2 stages behind the next one under way, and counts on the last of these being issued by then.
    constexpr int READY = !FOLD ? UNITS - 2 : 3 * IB - 1 < UNITS - AHEAD ? 3 * IB - 1 : UNITS - AHEAD, FREE = UNITS - 1;
    constexpr int GAPS = FOLD ? JB : 2 * IB, ALL = COPIES + W_COPIES + S_COPIES, PIECES = 8 * JB / IB;
    static_assert(READY >= COPIED, "the wait counts whole stages");
    static_assert(!FOLD || (READY <= UNITS - AHEAD && UNITS % XR == 0), "no read in front of the barrier");
    auto copies_of = [&](int kt, int v, int gap) {
        const int third = v == FREE ? 0 : v + 1;         // (the last one in unit COPIED - 1)
        const int at = third * GAPS + gap, first = at * ALL / (3 * GAPS), last = (at + 1) * ALL / (3 * GAPS);
#pragma unroll
        for (int c = 0; c < ALL / (3 * GAPS) + 1; ++c)
            if (third < 3 && first + c < last) copy(v == FREE ? kt + NST : kt + NST - 1, first + c, v == FREE ? cur : prv);
    };
    // FOLD: a unit of work is one k-step of 32 columns and one row block: its JB matrix instructions and, between them, a share
    // of the widening of the next k-step's weights and the read of a row block some units ahead, so that LDS is read evenly.
    auto read = [&](int v) { x[v % XR] = row_block(v % IB, v / IB); };
    auto unit = [&](int kt, int v) {
        const int ks = v / IB, i = v % IB, nks = (ks + 1) & 3;
        read(v + AHEAD);
        if (ks % (4 / PER) == 0) fold(i, ks * PER / 4 - 1);
#pragma unroll
        for (int j = 0; j < JB; ++j) {
            const v4f zero = {};
            v4f& c = part[FOLD ? i : 0][FOLD ? j : 0];
            c = TY::mfma(b[ks & 1][j], x[v % XR], ks % (4 / PER) == 0 ? zero : c);
            copies_of(kt, v, j);
            if (!S_LDS && v >= 2 && v < 2 + JB && j == 0) fetch(kt + 1, v - 2);
#pragma unroll
            for (int p = i * PIECES + j * PIECES / JB; p < i * PIECES + (j + 1) * PIECES / JB; ++p) {
                const int block = p / 8;
                if (p % 8 == 0 && nks % (4 / PER) == 0) s[block].set(zero_of(block, nks * PER / 4));
                s[block].widen(p % 8, w[block], b[nks & 1][block], mask, bits, one);
            }
            if (i == IB - 1) w[j] = packed(j, ks + 2);   // (block j has been widened)
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Else: one k-step and one pair of channel blocks.  Between its 2 IB matrix instructions the next pair's weights are widened
    // and, in the k-step's last unit, the row blocks replaced by the next k-step's.  Sums are in units of their channel's scale:
    // unit_of, of channel l16 of block j; where a group begins they are multiplied by change, of channels 4 g .. 4 g + 3.
    // A scale of 0 leaves the unit as it is, and the group's weights are zeros.
    float unit_of[JB], change[2][2][4] = {};
#pragma unroll
    for (int j = 0; j < JB; ++j) unit_of[j] = 1.0f;
    bool off[JB];
    auto to_outputs = [&](float v, float (&out)[4]) {    // lane: of channel l16 -> of channels 4 g .. 4 g + 3
#pragma unroll
        for (int r = 0; r < 4; ++r) out[r] = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(16 * g + 4 * r, __builtin_bit_cast(int, v)));
    };
    auto begin_group = [&](int j, float (&by)[4]) {      // (a stage is a group)
        const float scale = (float)__builtin_bit_cast(_Float16, (uint16_t)sz[j]);
        off[j] = scale == 0.0f;
        const float to = off[j] ? unit_of[j] : scale, inverse = __builtin_amdgcn_rcpf(to);
        float ratio = unit_of[j] * inverse;              // one step on the division's remainder: 1 for equal scales
        ratio = __builtin_fmaf(__builtin_fmaf(-to, ratio, unit_of[j]), inverse, ratio);
        to_outputs(ratio, by);
        unit_of[j] = to;
        s[j].set(off[j] ? 0 : zero_of(j, 0));
    };
    auto pair = [&](int kt, int v) __attribute__((always_inline)) {
        const int ks = v / PAIRS, next = (v + 1) % UNITS, nks = next / PAIRS, nj = next % PAIRS * 2;
#pragma unroll
        for (int i = 0; i < IB; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = v % PAIRS * 2 + h, gap = i * 2 + h, block = gap / IB, piece = gap % IB;
                if (ks == 0) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] *= change[v & 1][h][r];
                }
                acc[i][j] = TY::mfma(b[v & 1][h], x[i % XR], acc[i][j]);
                copies_of(kt, v, gap);
                if (v == 2 && gap % (GAPS / JB) == 0) fetch(kt + 1, gap / (GAPS / JB));
                if (piece == 0) {
                    if (nks == 0) begin_group(nj + block, change[next & 1][block]);
                    if (off[nj + block]) w[block] = 0;
                }
                s[nj + block].widen(piece, w[block], b[next & 1][block], mask, bits, one);
                if (piece == 7) w[block] = packed((v + 2) % PAIRS * 2 + block, (v + 2) / PAIRS);
                if (h == 1 && v % PAIRS == PAIRS - 1) x[i % XR] = row_block(i, ks + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    auto work = [&](int kt, int v) __attribute__((always_inline)) {
        if constexpr (FOLD) unit(kt, v);
        else pair(kt, v);
    };
    if (kt_end) {
        if constexpr (!S_LDS) {
#pragma unroll
            for (int j = 0; j < JB; ++j) fetch(0, j);
        }
#pragma unroll
        for (int d = 0; d < NST - 1; ++d)
#pragma unroll
            for (int c = 0; c < ALL; ++c) copy(d, c, d * STAGE);
        gemm_dev::wait_stage<(NST - 2) * ALL>();
        __syncthreads();
        take(0);
#pragma unroll
        for (int c = 0; c < ALL / 3; ++c) copy(NST - 1, c, prv);
        if constexpr (FOLD) {
#pragma unroll
            for (int v = 0; v < AHEAD; ++v) read(v);
        } else {
#pragma unroll
            for (int i = 0; i < IB; ++i) x[i % XR] = row_block(i, 0);
        }
#pragma unroll
        for (int j = 0; j < WB; ++j) {
            w[j] = packed(j, 0);
            if constexpr (FOLD) {
                s[j].set(zero_of(j, 0));
            } else {
                begin_group(j, change[0][j]);
                if (off[j]) w[j] = 0;
            }
#pragma unroll
            for (int p = 0; p < 8; ++p) s[j].widen(p, w[j], b[0][j], mask, bits, one);
            w[j] = FOLD ? packed(j, 1) : packed(1 % PAIRS * 2 + j, 1 / PAIRS);
        }
    }
    constexpr int TAKE = FOLD ? 3 * IB : FREE;           // before this unit: the next stage's zero points and scales
    for (int kt = 0; kt < kt_end; ++kt) {
        if constexpr (FOLD) take_fold(cur);
#pragma unroll
        for (int v = 0; v < READY; ++v) work(kt, v);
        gemm_dev::wait_stage<(NST - 2) * ALL>();
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int v = READY; v < TAKE; ++v) work(kt, v);
        take(nxt);
#pragma unroll
        for (int v = TAKE; v < FREE; ++v) work(kt, v);
        gemm_dev::wait_stage<63>();
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        work(kt, FREE);
        prv = cur;
        cur = nxt;
        nxt = nxt + STAGE == NST * STAGE ? 0 : nxt + STAGE;
    }
    gemm_dev::wait_vm<0>();                              // (the copies beyond the end)
    if constexpr (FOLD) {
#pragma unroll
        for (int i = 0; i < IB; ++i) fold(i, PER - 1);
    } else {                                             // (the first pair has its units for the stage beyond the end)
#pragma unroll
        for (int j = 0; j < JB; ++j) {
            float units[4];
            to_outputs(unit_of[j], units);
#pragma unroll
            for (int i = 0; i < IB; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][r] = (j < 2 ? acc[i][j][r] * change[0][j & 1][r] : acc[i][j][r]) * units[r];
        }
    }
    if constexpr (KS > 1) {
        __syncthreads();
        float4* const red = reinterpret_cast<float4*>(all_lds);
        if (kg > 0) {
#pragma unroll
            for (int i = 0; i < IB; ++i)
#pragma unroll
                for (int j = 0; j < JB; ++j)
                    red[(((kg - 1) * NW + wave) * IB * JB + i * JB + j) * 64 + lane] = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int k = 0; k < KS - 1; ++k)
#pragma unroll
            for (int i = 0; i < IB; ++i)
#pragma unroll
                for (int j = 0; j < JB; ++j) {
                    const float4 f = red[((k * NW + wave) * IB * JB + i * JB + j) * 64 + lane];
                    acc[i][j][0] += f.x; acc[i][j][1] += f.y; acc[i][j][2] += f.z; acc[i][j][3] += f.w;
                }
    }

    // ---- lane: row l16 of every row block, channels 4 g .. 4 g + 3 of every channel block
    const bool wide = a.ldy % 4 == 0 && (reinterpret_cast<uintptr_t>(a.y) & 7) == 0;
#pragma unroll
    for (int i = 0; i < IB; ++i) {
        const int r = (wm * IB + i) * 16 + l16;
        if (r >= src.count) continue;
        const size_t row = list ? (size_t)list[r] : (size_t)src.first + r;
#pragma unroll
        for (int j = 0; j < JB; ++j) {
            if (a.glu && j % 2) continue;
            const int block = b0 + wn * JB + j, n = (a.glu ? block >> 1 : block) * kBlock + 4 * g;
            if (n >= a.width) continue;
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int nq = min(n + q, a.width - 1);
                v[q] = acc[i][j][q];
                if (src.expert < 0) { v[q] = 0.0f; continue; }
                if (a.bias) v[q] += TY::load(a.bias, e * a.w.N + nq);
                if (a.glu) {
                    float u = acc[i][j + 1 < JB ? j + 1 : j][q];
                    if (a.bias) u += TY::load(a.bias, e * a.w.N + a.width + nq);
                    v[q] = silu_product(v[q], u);
                }
            }
            if (a.weights) {
                float* to = a.stage + row * a.width + n;
                if (n + 3 < a.width && a.width % 4 == 0) *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
                else for (int q = 0; q < 4 && n + q < a.width; ++q) to[q] = v[q];
            } else {
                uint16_t* to = static_cast<uint16_t*>(a.y) + row * a.ldy + n;
                if (wide && n + 3 < a.width)
                    *reinterpret_cast<uint2*>(to) = make_uint2(TY::round(v[0]) | (uint32_t)TY::round(v[1]) << 16,
                                                               TY::round(v[2]) | (uint32_t)TY::round(v[3]) << 16);
                else
                    for (int q = 0; q < 4 && n + q < a.width; ++q) to[q] = TY::round(v[q]);
            }
        }
    }
}

template <typename TY, int KG, int IB, int JB, int WM, int WN, int KS, int NST, int OCC, bool FOLD>
hipError_t launch_tiles(const W4gArgs& a, hipStream_t stream) {
    const int bm = IB * WM * 16, tiles_m = a.ids ? a.rows / bm + min(a.rows, a.experts + 1) : (a.rows + bm - 1) / bm;
    const int tiles_n = (a.w.nt + JB * WN - 1) / (JB * WN);
    hipLaunchKernelGGL((w4g_tiles_kernel<TY, KG, IB, JB, WM, WN, KS, NST, OCC, FOLD>), dim3((unsigned)tiles_m * tiles_n), dim3(WM * WN * KS * 64), 0, stream, a, tiles_m);
    return hipGetLastError();
}

}  // namespace

}  // namespace quik
