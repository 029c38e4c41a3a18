// Launch interfaces of the layers with 4-bit weights in groups and of the layers of experts (quik_w4g_api.hip is their
// C boundary).  Private to the shared library.
#pragma once
#include "quik_w4g_device.h"

namespace quik {

// One product of activations with w4g weights; `rows` rows of output before they are combined.
struct W4gArgs {
    const void* x;                // 16 bits [.., ldx]
    int ldx;
    w4g::Weights w;
    int group;                    // columns of a stored group: 32, 64 or 128
    int bf16, glu;                // type of x, bias and y; paired halves
    const void* bias;             // [E][N] or null
    void* y;                      // [.., ldy]
    int ldy;
    int width;                    // columns of y: N, or N / 2 for paired halves
    int rows;                     // dense: tokens; experts: T * top_k
    // experts only (ids == null: dense)
    const int32_t* ids;           // [rows]
    int experts, top_k;
    int x_per_slot;               // row r of x is r, else r / top_k
    int32_t* plan;                // room for launch_moe_plan's, which launch_w4g makes where it uses one
    const float* weights;         // [rows]: y is [T], the weighted sum of a token's slots; or null: y is [rows]
    float* stage;                 // [rows][width] for the sum, where the rows are computed one by one
};
hipError_t launch_w4g(const W4gArgs& a, hipStream_t stream);   // hipErrorInvalidConfiguration: more threads than a grid takes
// The kernels a product can run on: rows x channels of a workgroup's tile.  kW4gRows...: the waves split K (quik_w4g.hip);
// kW4gTile...: quik_w4g_tiles.hip
enum { kW4gRows16x16, kW4gRows16x32Wide, kW4gRows16x32, kW4gRows16x64, kW4gRows32x32, kW4gRows32x64,
       kW4gTile32x128, kW4gTile64x128, kW4gTile128x128, kW4gTile256x128, kW4gTile256x256,
       kW4gTile32x128Small, kW4gTile64x128Small, kW4gForms };    // (Small: several workgroups to a CU)
// What a product runs on (host only; launch_w4g launches exactly this): top_k, combine: experts' slots to a token, with weights;
// group: the stored one; experts: 0 for a dense layer
struct W4gChoice {
    int form;
    bool by_rows;                 // experts: a row at a time, without a plan
    bool by_token;                // of those: a token and the sum of its slots at a time
};
W4gChoice resolve_w4g(int rows, int top_k, bool combine, int blocks, int kt, int group, bool glu, int experts, int cus);
void set_w4g_form(int form);                                            // test hook: -1 automatic
hipError_t launch_w4g_tiles(const W4gArgs& a, int form, hipStream_t stream);
hipError_t launch_w4g_tiles256(const W4gArgs& a, hipStream_t stream);   // (groups of 128, dense, no paired halves)
hipError_t launch_weight_pack_w4g(const void* w_q, int ldw, const void* w_scale, const void* w_zero, int N, int K, int group,
                                  int glu, int experts, void* w4, hipStream_t stream);

// plan: int32 [experts + 2 + rows]: first row of every expert, the number of rows that have one, the number of rows; then
// the rows, ordered by expert, those of no expert last, in ascending order each
hipError_t launch_moe_plan(const int32_t* ids, int rows, int experts, int32_t* plan, hipStream_t stream);
hipError_t launch_moe_combine(const float* stage, const int32_t* ids, const float* weights, int T, int top_k, int experts,
                              int width, int bf16, void* y, int ldy, hipStream_t stream);

struct MoeRouteArgs {
    const void* logits;           // [T, ldl]
    int type;                     // QUIK_F16, QUIK_BF16, QUIK_F32
    int T, E, ldl;
    const float* bias;            // [E] or null
    int sigmoid;                  // else softmax
    int groups, topk_groups, group_top, top_k, renormalize;
    float scale;
    int32_t* ids;                 // [T, top_k]
    float* weights;               // [T, top_k]
};
hipError_t launch_moe_route(const MoeRouteArgs& a, hipStream_t stream);

}  // namespace quik
