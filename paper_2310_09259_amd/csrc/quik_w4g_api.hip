// C ABI of the layers with 4-bit weights in groups and of the layers of experts: argument validation and dispatch.  See
// include/quik.h for the contract of every entry point.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "quik.h"
#include "quik_w4g.h"

namespace {

constexpr int kMaxK = 32768, kMaxN = 1 << 20, kMaxTokens = 1 << 24, kMaxRows = 1 << 24, kMaxExperts = 1024, kMaxTopK = 32,
              kMaxGroups = 64;
// the kernels address x from a tile's first row (experts: from its start), and scales and zero points, by 32-bit offsets
constexpr int kMaxLdx = 1 << 22;
constexpr size_t kMaxOffset = 0xF0000000u;

inline bool aligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline int status(hipError_t rc) { return rc == hipSuccess ? QUIK_OK : QUIK_ELAUNCH; }
// of a product, which refuses what no grid holds before it launches anything
inline int product_status(hipError_t rc) { return rc == hipErrorInvalidConfiguration ? QUIK_EUNSUPPORTED : status(rc); }
inline size_t up256(size_t v) { return (v + 255u) & ~size_t(255); }

int check_weights(int N, int K, int group, int glu, int experts) {
    if (N <= 0 || K <= 0 || group < 0 || experts <= 0 || (glu != 0 && glu != 1) || (glu && N % 2)) return QUIK_EINVAL;
    if (group != 0 && group != 32 && group != 64 && group % 128) return QUIK_EUNSUPPORTED;
    if (K > kMaxK || K % 8 || N > kMaxN || experts > kMaxExperts) return QUIK_EUNSUPPORTED;
    return QUIK_OK;
}

// what the two products have in common
int check_product(int type, const void* x, int T, int K, int ldx, const void* w4, int group, int has_zero, int glu,
                  const void* bias, int N, int experts, const void* y, int ldy) {
    const int rc = check_weights(N, K, group, glu, experts);
    if (rc != QUIK_OK) return rc;
    if ((type != QUIK_F16 && type != QUIK_BF16) || (has_zero != 0 && has_zero != 1)) return QUIK_EINVAL;
    if (T <= 0 || ldx < K || ldy < (glu ? N / 2 : N)) return QUIK_EINVAL;
    if (!x || !w4 || !y) return QUIK_ENULL;
    if (T > kMaxTokens || ldx > kMaxLdx) return QUIK_EUNSUPPORTED;
    const quik::w4g::Layout l = quik::w4g::layout(N, K, group, has_zero != 0, glu != 0, experts);
    if (l.total - l.scales_at > kMaxOffset) return QUIK_EUNSUPPORTED;
    if (ldx % 8 || !aligned(x, 16) || !aligned(w4, 16) || !aligned(y, 2) || !aligned(bias, 2)) return QUIK_EALIGN;
    return QUIK_OK;
}

quik::W4gArgs product(int type, const void* x, int ldx, const void* w4, int group, int has_zero, int glu, const void* bias,
                      int N, int K, int experts, void* y, int ldy) {
    const quik::w4g::Layout l = quik::w4g::layout(N, K, group, has_zero != 0, glu != 0, experts);
    const uint8_t* const base = static_cast<const uint8_t*>(w4);
    quik::W4gArgs a{};
    a.x = x; a.ldx = ldx;
    a.w = {base, base + l.scales_at, has_zero ? base + l.zeros_at : nullptr, l.codes, l.scales, l.zeros, N, K, l.nt, l.kt};
    a.group = l.kg; a.bf16 = type == QUIK_BF16; a.glu = glu;
    a.bias = bias; a.y = y; a.ldy = ldy; a.width = glu ? N / 2 : N;
    return a;
}

struct MoeWorkspace { size_t plan, stage, total; };
MoeWorkspace moe_workspace(int T, int top_k, int width, int experts, int combine) {
    MoeWorkspace w;
    const size_t rows = (size_t)T * top_k;
    w.plan = 0;
    w.stage = up256((experts + 2 + rows) * sizeof(int32_t));
    w.total = w.stage + (combine ? up256(rows * width * sizeof(float)) : 0);
    return w;
}
int check_slots(int T, int top_k, int experts) {
    if (T <= 0 || top_k <= 0 || experts <= 0) return QUIK_EINVAL;
    if (experts > kMaxExperts || top_k > kMaxTopK || T > kMaxRows / top_k) return QUIK_EUNSUPPORTED;
    return QUIK_OK;
}

}  // namespace

extern "C" {

size_t quik_w4g_bytes(int N, int K, int group, int has_zero, int glu, int experts) {
    if (check_weights(N, K, group, glu, experts) != QUIK_OK || (has_zero != 0 && has_zero != 1)) return 0;
    return quik::w4g::layout(N, K, group, has_zero != 0, glu != 0, experts).total;
}

int quik_weight_pack_w4g(const void* w_q, int ldw, const void* w_scale, const void* w_zero, int N, int K, int group, int glu,
                         int experts, void* w4, void* stream) {
    const int rc = check_weights(N, K, group, glu, experts);
    if (rc != QUIK_OK) return rc;
    if (ldw < K / 2) return QUIK_EINVAL;
    if (!w_q || !w_scale || !w4) return QUIK_ENULL;
    if (ldw % 16 || !aligned(w_q, 16) || !aligned(w4, 16) || !aligned(w_scale, 2)) return QUIK_EALIGN;
    return status(quik::launch_weight_pack_w4g(w_q, ldw, w_scale, w_zero, N, K, group, glu, experts, w4,
                                               static_cast<hipStream_t>(stream)));
}

int quik_linear_w4g(int type, const void* x, int T, int K, int ldx, const void* w4, int group, int has_zero, int glu,
                    const void* bias, int N, void* y, int ldy, void* stream) {
    const int rc = check_product(type, x, T, K, ldx, w4, group, has_zero, glu, bias, N, 1, y, ldy);
    if (rc != QUIK_OK) return rc;
    quik::W4gArgs a = product(type, x, ldx, w4, group, has_zero, glu, bias, N, K, 1, y, ldy);
    a.rows = T;
    return product_status(quik::launch_w4g(a, static_cast<hipStream_t>(stream)));
}

int quik_debug_w4g_form(int rows, int N, int K, int glu, int experts, int cus) {
    if (rows <= 0 || experts < 0 || cus <= 0) return QUIK_EINVAL;
    const int rc = check_weights(N, K, 0, glu, experts ? experts : 1);
    if (rc != QUIK_OK) return rc;
    const quik::w4g::Layout l = quik::w4g::layout(N, K, 0, false, glu != 0, 1);
    return quik::resolve_w4g(rows, 1, false, l.nt, l.kt, l.kg, glu != 0, experts, cus).form;
}

int quik_debug_moe_w4g_form(int T, int top_k, int N, int K, int group, int glu, int experts, int combine, int cus) {
    int rc = check_slots(T, top_k, experts);
    if (rc != QUIK_OK) return rc;
    if ((combine != 0 && combine != 1) || cus <= 0) return QUIK_EINVAL;
    rc = check_weights(N, K, group, glu, experts);
    if (rc != QUIK_OK) return rc;
    const quik::w4g::Layout l = quik::w4g::layout(N, K, group, false, glu != 0, 1);
    return quik::resolve_w4g(T * top_k, top_k, combine != 0, l.nt, l.kt, l.kg, glu != 0, experts, cus).form;
}

int quik_debug_set_w4g_form(int form) {
    if (form < -1 || form >= quik::kW4gForms) return QUIK_EINVAL;
    quik::set_w4g_form(form);
    return QUIK_OK;
}

int quik_moe_route(int type, const void* logits, int T, int experts, int ldl, const float* bias, int score, int groups,
                   int topk_groups, int group_top, int top_k, int renormalize, float scale, int32_t* ids, float* weights,
                   void* stream) {
    if (type != QUIK_F16 && type != QUIK_BF16 && type != QUIK_F32) return QUIK_EINVAL;
    if (score != QUIK_SOFTMAX && score != QUIK_SIGMOID) return QUIK_EINVAL;
    if (renormalize != 0 && renormalize != 1) return QUIK_EINVAL;
    const int rc = check_slots(T, top_k, experts);
    if (rc != QUIK_OK) return rc;
    if (ldl < experts || top_k > experts || groups <= 0 || experts % groups) return QUIK_EINVAL;
    const int size = experts / groups;
    if (topk_groups <= 0 || topk_groups > groups || group_top <= 0 || group_top > size || top_k > topk_groups * size) return QUIK_EINVAL;
    if (!logits || !ids || !weights) return QUIK_ENULL;
    if (groups > kMaxGroups) return QUIK_EUNSUPPORTED;
    if (!aligned(logits, type == QUIK_F32 ? 4 : 2) || !aligned(bias, 4) || !aligned(ids, 4) || !aligned(weights, 4)) return QUIK_EALIGN;
    const quik::MoeRouteArgs a{logits, type, T, experts, ldl, bias, score == QUIK_SIGMOID, groups, topk_groups, group_top, top_k,
                               renormalize, scale, ids, weights};
    return status(quik::launch_moe_route(a, static_cast<hipStream_t>(stream)));
}

size_t quik_moe_workspace_bytes(int T, int top_k, int N, int glu, int experts, int combine) {
    if (N <= 0 || N > kMaxN || (glu != 0 && glu != 1) || (glu && N % 2) || check_slots(T, top_k, experts) != QUIK_OK) return 0;
    return moe_workspace(T, top_k, glu ? N / 2 : N, experts, combine).total;
}

int quik_moe_linear_w4g(int type, const void* x, int ldx, int x_per_slot, const int32_t* ids, const float* weights, int T,
                        int top_k, int K, const void* w4, int group, int has_zero, int glu, const void* bias, int N,
                        int experts, void* y, int ldy, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_slots(T, top_k, experts);
    if (rc != QUIK_OK) return rc;
    rc = check_product(type, x, T, K, ldx, w4, group, has_zero, glu, bias, N, experts, y, ldy);
    if (rc != QUIK_OK) return rc;
    if (x_per_slot != 0 && x_per_slot != 1) return QUIK_EINVAL;
    if ((size_t)T * (x_per_slot ? top_k : 1) * ldx * 2 > kMaxOffset) return QUIK_EUNSUPPORTED;
    if (!ids || !workspace) return QUIK_ENULL;
    if (!aligned(ids, 4) || !aligned(weights, 4) || !aligned(workspace, 256)) return QUIK_EALIGN;
    const MoeWorkspace m = moe_workspace(T, top_k, glu ? N / 2 : N, experts, weights != nullptr);
    if (workspace_bytes < m.total) return QUIK_EWORKSPACE;
    uint8_t* const base = static_cast<uint8_t*>(workspace);
    quik::W4gArgs a = product(type, x, ldx, w4, group, has_zero, glu, bias, N, K, experts, y, ldy);
    a.rows = T * top_k;
    a.ids = ids; a.experts = experts; a.top_k = top_k; a.x_per_slot = x_per_slot;
    a.weights = weights;
    a.plan = reinterpret_cast<int32_t*>(base + m.plan);
    a.stage = weights ? reinterpret_cast<float*>(base + m.stage) : nullptr;
    return product_status(quik::launch_w4g(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
