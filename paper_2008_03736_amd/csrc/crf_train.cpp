// crf_train.cpp -- C entry points of the fine-tuning operators: argument
// checks and launches, as crf_plan.cpp has them for the others.
#include <hip/hip_runtime_api.h>

#include <atomic>
#include <cstring>

#include "../../include/crf_inside.h"
#include "crf_plan.h"

using crf::check_device;
using crf::fail;
using crf::hip_fail;
using crf::ok;

namespace {

// Finite and at least 0, by the bits: the build takes no account of NaN in
// comparisons.
bool finite_positive(float x) {
    uint32_t u;
    std::memcpy(&u, &x, 4);
    return u < 0x7F800000u || u == 0x80000000u;
}

bool misaligned(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

int check_workspace(const void *workspace, int64_t have, int64_t need) {
    if (workspace == nullptr) return fail(CRF_EINVAL, "workspace is NULL");
    if (misaligned(workspace, 256)) return fail(CRF_EINVAL, "workspace must be 256-byte aligned");
    if (have < need)
        return fail(CRF_EINVAL, "workspace of %lld bytes, %lld are needed", (long long)have, (long long)need);
    return CRF_OK;
}

int64_t tree_bytes(const crf_plan *plan) { return ((int64_t)plan->B * 8 + 255) / 256 * 256; }

// What the tree calls have in common.
int check_trees(const crf_plan *plan, const int32_t *trees, int32_t num_trees) {
    if (num_trees < 1 || num_trees > CRF_MAX_TREES)
        return fail(CRF_EINVAL, "num_trees %d outside [1, %d]", num_trees, CRF_MAX_TREES);
    if (misaligned(trees, 8)) return fail(CRF_EINVAL, "trees must be 8-byte aligned");
    if (plan->L != 1) return fail(CRF_EUNSUPPORTED, "trees of labelled scores (L = %d)", plan->L);
    return CRF_OK;
}

int check_row(int32_t d) {
    if (d < 4 || d > CRF_MAX_ROW || d % 4 != 0)
        return fail(CRF_EINVAL, "d %d is not a multiple of 4 in [4, %d]", d, CRF_MAX_ROW);
    return CRF_OK;
}

int check_scorer(int32_t d, int32_t ldw, int32_t num_labels) {
    if (d < 4 || d > crf::kBiaMaxD || d % 4 != 0)
        return fail(CRF_EINVAL, "d %d is not a multiple of 4 in [4, %d]", d, crf::kBiaMaxD);
    if (ldw < d + 1 || ldw % 4 != 0) return fail(CRF_EINVAL, "ldw %d < d+1 or not a multiple of 4", ldw);
    if (num_labels < 1 || num_labels > CRF_MAX_LABELS)
        return fail(CRF_EINVAL, "num_labels %d outside [1, %d]", num_labels, CRF_MAX_LABELS);
    return CRF_OK;
}

// crf_biaffine_bwd and crf_biaffine_bwd_packed once rl and rr are checked.
int scorer_backward(const crf_plan *plan, const void *rl, const uint8_t *rl_scales, const void *rr,
                    const uint8_t *rr_scales, const uint16_t *w, int32_t d, int32_t ldw, int32_t num_labels,
                    const float *grad_scores, uint16_t *grad_rl, uint16_t *grad_rr, float *grad_w, void *workspace,
                    int64_t workspace_bytes, void *stream, const char *what) {
    int rc = check_scorer(d, ldw, num_labels);
    if (rc != CRF_OK) return rc;
    if (misaligned(grad_rl, 8) || misaligned(grad_rr, 8)) return fail(CRF_EINVAL, "grad_rl/grad_rr must be 8-byte aligned");
    if (misaligned(grad_w, 16)) return fail(CRF_EINVAL, "grad_w must be 16-byte aligned");
    const void *ins[] = {rl, rr, rl_scales, rr_scales, w, grad_scores};
    const void *outs[] = {grad_rl, grad_rr, grad_w};
    for (const void *o : outs)
        for (const void *i : ins)
            if (o != nullptr && o == i) return fail(CRF_EINVAL, "a gradient must not alias an input");
    if (grad_rl != nullptr && grad_rl == grad_rr) return fail(CRF_EINVAL, "grad_rl and grad_rr must not alias");
    if ((rc = check_workspace(workspace, workspace_bytes, crf::biaffine_bwd_bytes(plan->kp, plan->cells, d, num_labels))) !=
            CRF_OK ||
        (rc = check_device(plan)) != CRF_OK)
        return rc;
    // best effort, as for the other kernels: a real shortfall surfaces as a launch error
    static std::atomic<uint64_t> seen{0};
    const uint64_t bit = (uint64_t)1 << (plan->device & 63);
    if (!(seen.fetch_or(bit) & bit) && crf::set_biaffine_bwd_attributes() != hipSuccess) (void)hipGetLastError();
    const hipError_t e = crf::launch_biaffine_bwd(plan->kp, plan->cells, rl, rl_scales, rr, rr_scales, w, d, ldw, num_labels,
                                                  grad_scores, grad_rl, grad_rr, grad_w, static_cast<char *>(workspace),
                                                  static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, what);
}

}  // namespace

extern "C" {

int crf_tree_workspace(const crf_plan *plan, int64_t *bytes) {
    if (plan == nullptr || bytes == nullptr) return fail(CRF_EINVAL, "NULL argument");
    *bytes = tree_bytes(plan);
    return ok();
}

int crf_tree_logprobs(const crf_plan *plan, const float *scores, const int32_t *trees, int32_t num_trees,
                      const int32_t *counts, float *logp, float *logZ, void *workspace, int64_t workspace_bytes,
                      void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (scores == nullptr || trees == nullptr || logp == nullptr)
        return fail(CRF_EINVAL, "scores/trees/logp is NULL");
    int rc = check_trees(plan, trees, num_trees);
    if (rc != CRF_OK || (rc = check_workspace(workspace, workspace_bytes, tree_bytes(plan))) != CRF_OK ||
        (rc = check_device(plan)) != CRF_OK)
        return rc;
    const hipError_t e = crf::launch_tree_logprobs(plan->kp, scores, trees, num_trees, counts,
                                                   static_cast<double *>(workspace), logp, logZ,
                                                   static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_tree_logprobs launch");
}

int crf_tree_logprobs_bwd(const crf_plan *plan, const float *scores, const int32_t *trees, int32_t num_trees,
                          const int32_t *counts, const float *grad_logp, float *grad_scores, void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (scores == nullptr || trees == nullptr || grad_logp == nullptr || grad_scores == nullptr)
        return fail(CRF_EINVAL, "scores/trees/grad_logp/grad_scores is NULL");
    if (scores == grad_scores) return fail(CRF_EINVAL, "grad_scores must not alias scores");
    int rc = check_trees(plan, trees, num_trees);
    if (rc != CRF_OK || (rc = check_device(plan)) != CRF_OK) return rc;
    const hipError_t e = crf::launch_tree_logprobs_bwd(plan->kp, scores, trees, num_trees, counts,
                                                       grad_logp, grad_scores, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_tree_logprobs_bwd launch");
}

int crf_policy_loss(const crf_plan *plan, const float *scores, const int32_t *trees, int32_t num_trees,
                    const int32_t *counts, const float *advantages, const float *old_logp, const float *ref_logp,
                    float clip_low, float clip_high, float kl_coef, const float *grad_loss, float *loss, float *logp,
                    float *grad_scores, void *workspace, int64_t workspace_bytes, void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (scores == nullptr || trees == nullptr || advantages == nullptr || old_logp == nullptr || loss == nullptr ||
        grad_scores == nullptr)
        return fail(CRF_EINVAL, "scores/trees/advantages/old_logp/loss/grad_scores is NULL");
    if (scores == grad_scores) return fail(CRF_EINVAL, "grad_scores must not alias scores");
    // (a long sentence's stripes each read them, and the first one writes)
    const float *ins[] = {advantages, old_logp, ref_logp, grad_loss};
    for (const float *in : ins)
        if (in != nullptr && (in == loss || in == logp)) return fail(CRF_EINVAL, "loss and logp must not alias an input");
    if (!finite_positive(clip_low) || clip_low > 1.f)
        return fail(CRF_EINVAL, "clip_low %g outside [0, 1]", (double)clip_low);
    if (!finite_positive(clip_high))
        return fail(CRF_EINVAL, "clip_high %g is negative or not finite", (double)clip_high);
    if (!finite_positive(kl_coef)) return fail(CRF_EINVAL, "kl_coef %g is negative or not finite", (double)kl_coef);
    if (kl_coef != 0.f && ref_logp == nullptr) return fail(CRF_EINVAL, "kl_coef %g without ref_logp", (double)kl_coef);
    int rc = check_trees(plan, trees, num_trees);
    if (rc != CRF_OK || (rc = check_workspace(workspace, workspace_bytes, tree_bytes(plan))) != CRF_OK ||
        (rc = check_device(plan)) != CRF_OK)
        return rc;
    const hipError_t e = crf::launch_policy_loss(plan->kp, scores, trees, num_trees, counts, advantages,
                                                 old_logp, ref_logp, clip_low, clip_high, kl_coef, grad_loss,
                                                 static_cast<double *>(workspace), loss, logp, grad_scores,
                                                 static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_policy_loss launch");
}

int crf_pack_rows(const crf_plan *plan, const uint16_t *x, int32_t d, uint8_t *codes, uint8_t *scales, void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (x == nullptr || codes == nullptr || scales == nullptr) return fail(CRF_EINVAL, "x/codes/scales is NULL");
    int rc = check_row(d);
    if (rc != CRF_OK) return rc;
    if (misaligned(x, 8)) return fail(CRF_EINVAL, "x must be 8-byte aligned");
    if (misaligned(codes, 16)) return fail(CRF_EINVAL, "codes must be 16-byte aligned");
    if (static_cast<const void *>(x) == codes) return fail(CRF_EINVAL, "x and codes must not alias");
    if ((rc = check_device(plan)) != CRF_OK) return rc;
    const hipError_t e = crf::launch_pack_rows(plan->kp, x, d, codes, scales, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_pack_rows launch");
}

int crf_unpack_rows(const crf_plan *plan, const uint8_t *codes, const uint8_t *scales, int32_t d, uint16_t *x,
                    void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (x == nullptr || codes == nullptr || scales == nullptr) return fail(CRF_EINVAL, "codes/scales/x is NULL");
    int rc = check_row(d);
    if (rc != CRF_OK) return rc;
    if (misaligned(x, 8)) return fail(CRF_EINVAL, "x must be 8-byte aligned");
    if (misaligned(codes, 16)) return fail(CRF_EINVAL, "codes must be 16-byte aligned");
    if (static_cast<const void *>(x) == codes) return fail(CRF_EINVAL, "x and codes must not alias");
    if ((rc = check_device(plan)) != CRF_OK) return rc;
    const hipError_t e = crf::launch_unpack_rows(plan->kp, codes, scales, d, x, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_unpack_rows launch");
}

int crf_biaffine_bwd_workspace(const crf_plan *plan, int32_t d, int32_t num_labels, int64_t *bytes) {
    if (plan == nullptr || bytes == nullptr) return fail(CRF_EINVAL, "NULL argument");
    const int rc = check_scorer(d, (d + 4) / 4 * 4, num_labels);
    if (rc != CRF_OK) return rc;
    *bytes = crf::biaffine_bwd_bytes(plan->kp, plan->cells, d, num_labels);
    return ok();
}

int crf_biaffine_bwd(const crf_plan *plan, const uint16_t *rl, const uint16_t *rr, const uint16_t *w, int32_t d,
                     int32_t ldw, int32_t num_labels, const float *grad_scores, uint16_t *grad_rl, uint16_t *grad_rr,
                     float *grad_w, void *workspace, int64_t workspace_bytes, void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (rl == nullptr || rr == nullptr || w == nullptr || grad_scores == nullptr)
        return fail(CRF_EINVAL, "rl/rr/w/grad_scores is NULL");
    if (misaligned(rl, 8) || misaligned(rr, 8) || misaligned(w, 8))
        return fail(CRF_EINVAL, "rl/rr/w must be 8-byte aligned");
    return scorer_backward(plan, rl, nullptr, rr, nullptr, w, d, ldw, num_labels, grad_scores, grad_rl, grad_rr, grad_w,
                           workspace, workspace_bytes, stream, "crf_biaffine_bwd launch");
}

int crf_biaffine_bwd_packed(const crf_plan *plan, const uint8_t *rl_codes, const uint8_t *rl_scales,
                            const uint8_t *rr_codes, const uint8_t *rr_scales, const uint16_t *w, int32_t d, int32_t ldw,
                            int32_t num_labels, const float *grad_scores, uint16_t *grad_rl, uint16_t *grad_rr,
                            float *grad_w, void *workspace, int64_t workspace_bytes, void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (rl_codes == nullptr || rl_scales == nullptr || rr_codes == nullptr || rr_scales == nullptr || w == nullptr ||
        grad_scores == nullptr)
        return fail(CRF_EINVAL, "rl_codes/rl_scales/rr_codes/rr_scales/w/grad_scores is NULL");
    if (misaligned(rl_codes, 16) || misaligned(rr_codes, 16))
        return fail(CRF_EINVAL, "rl_codes/rr_codes must be 16-byte aligned");
    if (misaligned(w, 8)) return fail(CRF_EINVAL, "w must be 8-byte aligned");
    return scorer_backward(plan, rl_codes, rl_scales, rr_codes, rr_scales, w, d, ldw, num_labels, grad_scores, grad_rl,
                           grad_rr, grad_w, workspace, workspace_bytes, stream, "crf_biaffine_bwd_packed launch");
}

}  // extern "C"
