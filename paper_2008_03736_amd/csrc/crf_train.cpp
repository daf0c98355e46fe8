// crf_train.cpp -- C entry points of the fine-tuning operators: argument
// checks and launches, as crf_plan.cpp has them for the others.
#include <hip/hip_runtime_api.h>

#include <cstring>
#include <initializer_list>
#include <mutex>

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

// A buffer of a call.
struct Span {
    const char *name;
    const void *at;   // NULL: not given
    int64_t bytes;
};
bool overlap(const Span &a, const Span &b) {
    const uintptr_t x = (uintptr_t)a.at, y = (uintptr_t)b.at;
    return x != 0 && y != 0 && x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}
// No output (the workspace is one) may share a byte with an input or another
// output: a call's workgroups read inputs while others write.
int check_overlap(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
    for (const Span *o = outs.begin(); o != outs.end(); ++o) {
        for (const Span &i : ins)
            if (overlap(*o, i)) return fail(CRF_EINVAL, "%s must not alias %s", o->name, i.name);
        for (const Span *q = outs.begin(); q != o; ++q)
            if (overlap(*o, *q)) return fail(CRF_EINVAL, "%s and %s must not alias", q->name, o->name);
    }
    return CRF_OK;
}
// Bytes of the arrays that calls share.
int64_t scores_bytes(const crf_plan *p, int64_t num_labels) { return 4 * num_labels * p->B * p->n1 * p->n1; }
int64_t trees_bytes(const crf_plan *p, int64_t num_trees) { return 8 * num_trees * p->B * (2 * (p->n1 - 1) - 1); }
int64_t rows_bytes(const crf_plan *p, int64_t entry, int64_t per_row) { return entry * per_row * p->B * p->n1; }
int64_t vec_bytes(const crf_plan *p) { return 4 * (int64_t)p->B; }
int64_t row_codes(int64_t d) { return (d + 31) / 32 * 32; }

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
    const int64_t need = crf::biaffine_bwd_bytes(plan->kp, plan->cells, d, num_labels);
    const int64_t bf16 = rows_bytes(plan, 2, d), w_entries = (int64_t)num_labels * d * ldw;
    const int64_t rows = rl_scales != nullptr ? rows_bytes(plan, 1, row_codes(d)) : bf16;
    const int64_t scales = rows_bytes(plan, 1, row_codes(d) / 32);
    if ((rc = check_workspace(workspace, workspace_bytes, need)) != CRF_OK ||
        (rc = check_overlap({{"grad_rl", grad_rl, bf16}, {"grad_rr", grad_rr, bf16}, {"grad_w", grad_w, 4 * w_entries},
                             {"workspace", workspace, need}},
                            {{"rl", rl, rows}, {"rr", rr, rows}, {"rl_scales", rl_scales, scales},
                             {"rr_scales", rr_scales, scales}, {"w", w, 2 * w_entries},
                             {"grad_scores", grad_scores, scores_bytes(plan, num_labels)}})) != CRF_OK ||
        (rc = check_device(plan)) != CRF_OK)
        return rc;
    // Once a device, and before any thread's first launch there: another one's
    // first call waits.  Best effort, as for the other kernels: a real shortfall
    // surfaces as a launch error.
    static std::once_flag set[64];
    std::call_once(set[plan->device & 63], [] {
        if (crf::set_biaffine_bwd_attributes() != hipSuccess) (void)hipGetLastError();
    });
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
    if (rc != CRF_OK) return rc;
    const int64_t each = num_trees * vec_bytes(plan);
    if ((rc = check_workspace(workspace, workspace_bytes, tree_bytes(plan))) != CRF_OK ||
        (rc = check_overlap({{"logp", logp, each}, {"logZ", logZ, vec_bytes(plan)}, {"workspace", workspace, tree_bytes(plan)}},
                            {{"scores", scores, scores_bytes(plan, 1)}, {"trees", trees, trees_bytes(plan, num_trees)},
                             {"counts", counts, vec_bytes(plan)}})) != CRF_OK ||
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
    int rc = check_trees(plan, trees, num_trees);
    if (rc != CRF_OK) return rc;
    if ((rc = check_overlap({{"grad_scores", grad_scores, scores_bytes(plan, 1)}},
                            {{"scores", scores, scores_bytes(plan, 1)}, {"trees", trees, trees_bytes(plan, num_trees)},
                             {"counts", counts, vec_bytes(plan)}, {"grad_logp", grad_logp, num_trees * vec_bytes(plan)}})) !=
            CRF_OK ||
        (rc = check_device(plan)) != CRF_OK)
        return rc;
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
    if (!finite_positive(clip_low) || clip_low > 1.f)
        return fail(CRF_EINVAL, "clip_low %g outside [0, 1]", (double)clip_low);
    if (!finite_positive(clip_high))
        return fail(CRF_EINVAL, "clip_high %g is negative or not finite", (double)clip_high);
    if (!finite_positive(kl_coef)) return fail(CRF_EINVAL, "kl_coef %g is negative or not finite", (double)kl_coef);
    if (kl_coef != 0.f && ref_logp == nullptr) return fail(CRF_EINVAL, "kl_coef %g without ref_logp", (double)kl_coef);
    int rc = check_trees(plan, trees, num_trees);
    if (rc != CRF_OK) return rc;
    const int64_t each = num_trees * vec_bytes(plan);
    if ((rc = check_workspace(workspace, workspace_bytes, tree_bytes(plan))) != CRF_OK ||
        (rc = check_overlap({{"loss", loss, vec_bytes(plan)}, {"logp", logp, each},
                             {"grad_scores", grad_scores, scores_bytes(plan, 1)},
                             {"workspace", workspace, tree_bytes(plan)}},
                            {{"scores", scores, scores_bytes(plan, 1)}, {"trees", trees, trees_bytes(plan, num_trees)},
                             {"counts", counts, vec_bytes(plan)}, {"advantages", advantages, each}, {"old_logp", old_logp, each},
                             {"ref_logp", ref_logp, each}, {"grad_loss", grad_loss, vec_bytes(plan)}})) != CRF_OK ||
        (rc = check_device(plan)) != CRF_OK)
        return rc;
    const hipError_t e = crf::launch_policy_loss(plan->kp, scores, trees, num_trees, counts, advantages,
                                                 old_logp, kl_coef != 0.f ? ref_logp : nullptr, clip_low, clip_high,
                                                 kl_coef, grad_loss,
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
    const Span rows[] = {{"x", x, rows_bytes(plan, 2, d)}, {"codes", codes, rows_bytes(plan, 1, row_codes(d))},
                         {"scales", scales, rows_bytes(plan, 1, row_codes(d) / 32)}};
    if ((rc = check_overlap({rows[1], rows[2]}, {rows[0]})) != CRF_OK || (rc = check_device(plan)) != CRF_OK) return rc;
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
    const Span rows[] = {{"x", x, rows_bytes(plan, 2, d)}, {"codes", codes, rows_bytes(plan, 1, row_codes(d))},
                         {"scales", scales, rows_bytes(plan, 1, row_codes(d) / 32)}};
    if ((rc = check_overlap({rows[0]}, {rows[1], rows[2]})) != CRF_OK || (rc = check_device(plan)) != CRF_OK) return rc;
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
