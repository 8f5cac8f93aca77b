// C ABI of what surrounds a layer that serves k experts per token: argument validation.  No kernel lives here.

#include <cmath>

#include "smoe_internal.h"

namespace {
constexpr int TOPK_MAX = 16, GROUPS_MAX = 16;

// T tokens of k choices each: the layer's per-token buffers hold one entry per pair.
int check_pairs(const smoe_layer* L, int T, int k, const char* who) {
    if (int rc = smoe_check_hot(L, T, who, false)) return rc;
    if (k < 1 || k > TOPK_MAX) return smoe_fail(SMOE_EINVAL, "%s: k=%d outside [1,%d]", who, k, TOPK_MAX);
    if ((int64_t)T * k > L->cfg.max_tokens)
        return smoe_fail(SMOE_EINVAL, "%s: T * k = %lld pairs exceed max_tokens=%d", who, (long long)T * k, L->cfg.max_tokens);
    return SMOE_OK;
}
}  // namespace

extern "C" {

size_t smoe_mx_scale_pitch(int d_model) { return d_model < 1 || d_model % 32 ? 0 : smoe_scale_pitch(d_model); }

int smoe_add_norm(smoe_layer_t* L, const void* x, const void* residual, const float* weight, float eps, int T, void* total, void* y,
                  void* q, void* q_scale, void* stream) {
    if (!L) return smoe_fail(SMOE_EINVAL, "smoe_add_norm: null handle");   // needs the handle's shape only: no bound workspace
    if (T < 0 || T > L->cfg.max_tokens) return smoe_fail(SMOE_EINVAL, "smoe_add_norm: T=%d outside [0,%d]", T, L->cfg.max_tokens);
    if (!(eps >= 0.f) || std::isinf(eps)) return smoe_fail(SMOE_EINVAL, "smoe_add_norm: eps must be a finite number >= 0");
    if (T == 0) return SMOE_OK;
    if (!x || !weight) return smoe_fail(SMOE_EINVAL, "smoe_add_norm: null input");
    if (!total && !y && !q) return smoe_fail(SMOE_EINVAL, "smoe_add_norm: no output");
    if (!q != !q_scale) return smoe_fail(SMOE_EINVAL, "smoe_add_norm: q and q_scale go together");
    if (q && L->cfg.d_model % 32) return smoe_fail(SMOE_EINVAL, "smoe_add_norm: 8-bit output needs d_model to be a multiple of 32");
    if (smoe_misaligned(x, 16) || smoe_misaligned(residual, 16) || smoe_misaligned(weight, 16) || smoe_misaligned(total, 16) ||
        smoe_misaligned(y, 16) || smoe_misaligned(q, 16) || smoe_misaligned(q_scale, 8))
        return smoe_fail(SMOE_EINVAL, "smoe_add_norm: rows and weight must be 16-byte aligned, scales 8-byte");
    return smoe_launch_add_norm(L, x, residual, weight, eps, T, total, y, q, q_scale, (hipStream_t)stream);
}

int smoe_route_topk(smoe_layer_t* L, const smoe_topk_rule* rule, const float* bias, const void* x, int T, int32_t* orig_expert,
                    float* orig_gate, int32_t* slot, float* gate, float* xnorm, void* stream) {
    if (!rule) return smoe_fail(SMOE_EINVAL, "smoe_route_topk: null rule");
    const smoe_topk_rule& r = *rule;
    if (int rc = check_pairs(L, T, r.k, "smoe_route_topk")) return rc;
    const smoe_config& c = L->cfg;
    if (r.score != SMOE_SCORE_SOFTMAX && r.score != SMOE_SCORE_SIGMOID)
        return smoe_fail(SMOE_EINVAL, "smoe_route_topk: unknown score %d", r.score);
    if (r.groups < 1 || r.groups > GROUPS_MAX || c.E % r.groups)
        return smoe_fail(SMOE_EINVAL, "smoe_route_topk: groups=%d is not a divisor of E=%d in [1,%d]", r.groups, c.E, GROUPS_MAX);
    if (r.groups_kept < 1 || r.groups_kept > r.groups)
        return smoe_fail(SMOE_EINVAL, "smoe_route_topk: groups_kept=%d outside [1,%d]", r.groups_kept, r.groups);
    if (r.group_best != 1 && r.group_best != 2)
        return smoe_fail(SMOE_EINVAL, "smoe_route_topk: group_best=%d is neither 1 nor 2", r.group_best);
    if (r.k > c.E / r.groups * r.groups_kept)
        return smoe_fail(SMOE_EINVAL, "smoe_route_topk: k=%d exceeds the %d experts of the kept groups", r.k, c.E / r.groups * r.groups_kept);
    if (r.renorm != 0 && r.renorm != 1) return smoe_fail(SMOE_EINVAL, "smoe_route_topk: renorm must be 0 or 1");
    if (!std::isfinite(r.scale)) return smoe_fail(SMOE_EINVAL, "smoe_route_topk: scale must be finite");
    if (int rc = smoe_check_hot(L, T, "smoe_route_topk", true)) return rc;
    if (T == 0) return SMOE_OK;
    if (!x || !orig_expert || !orig_gate || !slot || !gate || !xnorm) return smoe_fail(SMOE_EINVAL, "smoe_route_topk: null buffer");
    if (smoe_misaligned(x, 16)) return smoe_fail(SMOE_EINVAL, "smoe_route_topk: x must be 16-byte aligned");
    if (smoe_misaligned(bias, 4)) return smoe_fail(SMOE_EINVAL, "smoe_route_topk: bias must be 4-byte aligned");
    const hipStream_t s = (hipStream_t)stream;
    if (int rc = smoe_prepare_router(L, "smoe_route_topk", s)) return rc;
    if (int rc = smoe_once(L->router_norm, "smoe_route_topk", s, [&] { return smoe_launch_router_norm(L, s); })) return rc;
    return smoe_launch_route_topk(L, r, bias, x, T, orig_expert, orig_gate, slot, gate, xnorm, s);
}

int smoe_permute_topk(smoe_layer_t* L, const void* x, const int32_t* slot, int T, int k, void* x_perm, int32_t* perm, int32_t* inv_perm,
                      int32_t* offsets, void* stream) {
    if (int rc = check_pairs(L, T, k, "smoe_permute_topk")) return rc;
    if (!offsets) return smoe_fail(SMOE_EINVAL, "smoe_permute_topk: null offsets");
    if (T > 0 && (!slot || !perm || !inv_perm)) return smoe_fail(SMOE_EINVAL, "smoe_permute_topk: null buffer");
    if (T > 0 && x_perm && !x) return smoe_fail(SMOE_EINVAL, "smoe_permute_topk: x_perm without x");
    if (smoe_misaligned(x, 16) || smoe_misaligned(x_perm, 16))
        return smoe_fail(SMOE_EINVAL, "smoe_permute_topk: x and x_perm must be 16-byte aligned");
    return smoe_launch_permute_topk(L, x, slot, T, k, x_perm, perm, inv_perm, offsets, (hipStream_t)stream);
}

int smoe_expert_ffn_mx(smoe_layer_t* L, const void* q, const void* q_scale, const int32_t* perm, int k, const int32_t* offsets, int T,
                       void* y_perm, void* stream) {
    if (int rc = check_pairs(L, T, k, "smoe_expert_ffn_mx")) return rc;
    if (L->cfg.dtype != SMOE_MXFP8) return smoe_fail(SMOE_EINVAL, "smoe_expert_ffn_mx: only layers with 8-bit slots (SMOE_MXFP8)");
    if (!perm && k != 1) return smoe_fail(SMOE_EINVAL, "smoe_expert_ffn_mx: without perm row r is token r, which takes k = 1");
    if (int rc = smoe_check_hot(L, T, "smoe_expert_ffn_mx", true)) return rc;
    if (T == 0) return SMOE_OK;
    if (!q || !q_scale || !offsets || !y_perm) return smoe_fail(SMOE_EINVAL, "smoe_expert_ffn_mx: null buffer");
    if (smoe_misaligned(q, 16) || smoe_misaligned(q_scale, 8) || smoe_misaligned(y_perm, 16))
        return smoe_fail(SMOE_EINVAL, "smoe_expert_ffn_mx: q and y_perm must be 16-byte aligned, scales 8-byte");
    const int rc = smoe_launch_ffn_mx(L, q, q_scale, perm, k, offsets, T, y_perm, (hipStream_t)stream);
    smoe_note_slot_pass(L);
    L->prof_ev[0] = L->prof_ev[1] = L->prof_ev[2] = L->prof_ev[3] = nullptr;
    return rc;
}

int smoe_combine_topk(smoe_layer_t* L, const void* y_perm, const int32_t* inv_perm, const float* gate, const void* residual, int T, int k,
                      void* out, void* stream) {
    if (int rc = check_pairs(L, T, k, "smoe_combine_topk")) return rc;
    if (T == 0) return SMOE_OK;
    if (!y_perm || !inv_perm || !gate || !out) return smoe_fail(SMOE_EINVAL, "smoe_combine_topk: null buffer");
    if (smoe_misaligned(y_perm, 16) || smoe_misaligned(out, 16) || smoe_misaligned(residual, 16))
        return smoe_fail(SMOE_EINVAL, "smoe_combine_topk: y_perm, residual and out must be 16-byte aligned");
    return smoe_launch_combine_topk(L, y_perm, inv_perm, gate, residual, T, k, out, (hipStream_t)stream);
}

}  // extern "C"
