// crf_train.cpp -- C entry points of the operators that training a scorer and
// tuning a parser take: argument checks and launches, as crf_plan.cpp has them
// for the others.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
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

// Layer norm's rows: x is bf16 (8-byte aligned) or float32.
int check_norm(const void *x, int32_t x_type, int32_t d, float eps) {
    const int rc = check_row(d);
    if (rc != CRF_OK) return rc;
    if (x_type != CRF_BF16 && x_type != CRF_F32)
        return fail(CRF_EINVAL, "x_type %d is neither CRF_BF16 nor CRF_F32", x_type);
    if (misaligned(x, x_type == CRF_BF16 ? 8 : 4))
        return fail(CRF_EINVAL, "x must be %d-byte aligned", x_type == CRF_BF16 ? 8 : 4);
    // (squares beside a smaller one would be of few digits)
    if (!finite_positive(eps) || eps < FLT_MIN)
        return fail(CRF_EINVAL, "eps %g is not a finite number of 2^-126 or more", (double)eps);
    return CRF_OK;
}

int check_buckets(int32_t num_buckets, int32_t num_labels) {
    if (num_buckets < 1 || num_buckets > CRF_MAX_BUCKETS)
        return fail(CRF_EINVAL, "num_buckets %d outside [1, %d]", num_buckets, CRF_MAX_BUCKETS);
    if (num_labels < 1 || num_labels > CRF_MAX_LABELS)
        return fail(CRF_EINVAL, "num_labels %d outside [1, %d]", num_labels, CRF_MAX_LABELS);
    return CRF_OK;
}

int check_matrices(int32_t count, int32_t rows, int32_t cols, int32_t ld) {
    if (count < 1 || count > CRF_MAX_LABELS) return fail(CRF_EINVAL, "count %d outside [1, %d]", count, CRF_MAX_LABELS);
    if (rows < 1 || rows > CRF_MAX_ROW || cols < 1 || cols > CRF_MAX_ROW)
        return fail(CRF_EINVAL, "matrices of %d x %d, sides are in [1, %d]", rows, cols, CRF_MAX_ROW);
    if (ld < cols) return fail(CRF_EINVAL, "ld %d < cols %d", ld, cols);
    return CRF_OK;
}

// Once a device, before any thread's first launch there (see scorer_backward).
int set_update_attributes() {
    int device = 0;
    const hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
    static std::once_flag set[64];
    std::call_once(set[device & 63], [] {
        if (crf::set_ortho_attributes() != hipSuccess) (void)hipGetLastError();
    });
    return CRF_OK;
}

// What singular values, at most 1 at the start, grow to under the steps, and the
// polynomials that they are multiplied by: the kernels hold both in a float16's range.
int check_coefficients(const float *coefficients, int32_t steps, float eps) {
    if (coefficients == nullptr) return fail(CRF_EINVAL, "coefficients is NULL");
    if (steps < 1 || steps > CRF_MAX_STEPS) return fail(CRF_EINVAL, "steps %d outside [1, %d]", steps, CRF_MAX_STEPS);
    if (!finite_positive(eps) || eps == 0.f) return fail(CRF_EINVAL, "eps %g is not positive and finite", (double)eps);
    double most = 1.0;
    for (int k = 0; k < steps; ++k) {
        const float *f = coefficients + 3 * k;
        for (int q = 0; q < 3; ++q)
            if (!finite_positive(std::fabs(f[q])) || std::fabs(f[q]) > 1000.f)   // (no sum below overflows)
                return fail(CRF_EINVAL, "step %d's coefficient %g is outside [-1000, 1000]", k, (double)f[q]);
        const double a = f[0], b = f[1], c = f[2], top = most * most;   // t = s^2 in [0, top]
        auto value = [&](double t) { return std::sqrt(t) * std::fabs(a + t * (b + t * c)); };
        auto poly = [&](double t) { return std::fabs(a + t * (b + t * c)); };
        double grown = value(top), inner = std::max(poly(0.0), poly(top));
        auto at = [&](double t) {
            if (t > 0.0 && t < top) grown = std::max(grown, value(t)), inner = std::max(inner, poly(t));
        };
        // where a + 3 b t + 5 c t^2 is 0 (the larger root's numerator without a
        // difference, the other root from their product: c may be next to nothing
        // beside b), or b + 2 c t
        const double disc = 9.0 * b * b - 20.0 * a * c;
        if (disc >= 0.0) {
            const double sum = -0.5 * (3.0 * b + std::copysign(std::sqrt(disc), b));
            if (c != 0.0) at(sum / (5.0 * c));
            if (sum != 0.0) at(a / sum);
        }
        if (c != 0.0) at(-b / (2.0 * c));
        if (inner > 60.0 || grown > 4.0)
            return fail(CRF_EINVAL, "step %d takes singular values to %g (at most 4) by a polynomial of %g (at most 60)", k,
                        grown, inner);
        most = grown;
    }
    return CRF_OK;
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

int crf_layer_norm(const crf_plan *plan, const void *x, int32_t x_type, int32_t d, const float *gamma, const float *beta,
                   float eps, uint16_t *y, void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (x == nullptr || y == nullptr) return fail(CRF_EINVAL, "x/y is NULL");
    int rc = check_norm(x, x_type, d, eps);
    if (rc != CRF_OK) return rc;
    if (misaligned(y, 8)) return fail(CRF_EINVAL, "y must be 8-byte aligned");
    if ((rc = check_overlap({{"y", y, rows_bytes(plan, 2, d)}},
                            {{"x", x, rows_bytes(plan, x_type == CRF_F32 ? 4 : 2, d)}, {"gamma", gamma, 4 * (int64_t)d},
                             {"beta", beta, 4 * (int64_t)d}})) != CRF_OK ||
        (rc = check_device(plan)) != CRF_OK)
        return rc;
    const hipError_t e = crf::launch_norm(plan->kp, x, x_type == CRF_F32, d, gamma, beta, eps, y,
                                          static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_layer_norm launch");
}

int crf_layer_norm_bwd_workspace(const crf_plan *plan, int32_t d, int64_t *bytes) {
    if (plan == nullptr || bytes == nullptr) return fail(CRF_EINVAL, "NULL argument");
    const int rc = check_row(d);
    if (rc != CRF_OK) return rc;
    *bytes = crf::norm_bwd_bytes(plan->kp, d);
    return ok();
}

int crf_layer_norm_bwd(const crf_plan *plan, const void *x, int32_t x_type, int32_t d, const float *gamma,
                       const uint16_t *grad_y, float eps, void *grad_x, float *grad_gamma, float *grad_beta,
                       void *workspace, int64_t workspace_bytes, void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (x == nullptr || grad_y == nullptr) return fail(CRF_EINVAL, "x/grad_y is NULL");
    int rc = check_norm(x, x_type, d, eps);
    if (rc != CRF_OK) return rc;
    if (misaligned(grad_y, 8)) return fail(CRF_EINVAL, "grad_y must be 8-byte aligned");
    if (misaligned(grad_x, x_type == CRF_BF16 ? 8 : 4))
        return fail(CRF_EINVAL, "grad_x must be %d-byte aligned", x_type == CRF_BF16 ? 8 : 4);
    const int64_t need = crf::norm_bwd_bytes(plan->kp, d), own = rows_bytes(plan, x_type == CRF_F32 ? 4 : 2, d);
    const int64_t each = 4 * (int64_t)d;
    if ((rc = check_workspace(workspace, workspace_bytes, need)) != CRF_OK ||
        (rc = check_overlap({{"grad_x", grad_x, own}, {"grad_gamma", grad_gamma, each}, {"grad_beta", grad_beta, each},
                             {"workspace", workspace, need}},
                            {{"x", x, own}, {"gamma", gamma, each}, {"grad_y", grad_y, rows_bytes(plan, 2, d)}})) != CRF_OK ||
        (rc = check_device(plan)) != CRF_OK)
        return rc;
    if (grad_x == nullptr && grad_gamma == nullptr && grad_beta == nullptr) return ok();
    const hipError_t e = crf::launch_norm_bwd(plan->kp, x, x_type == CRF_F32, d, gamma, grad_y, eps, grad_x, grad_gamma,
                                              grad_beta, static_cast<char *>(workspace), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_layer_norm_bwd launch");
}

int crf_width_bias(const crf_plan *plan, const float *scores, int32_t num_labels, const float *table,
                   const int32_t *buckets, int32_t num_buckets, float *out, void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (scores == nullptr || table == nullptr || buckets == nullptr || out == nullptr)
        return fail(CRF_EINVAL, "scores/table/buckets/out is NULL");
    int rc = check_buckets(num_buckets, num_labels);
    if (rc != CRF_OK) return rc;
    const int64_t all = scores_bytes(plan, num_labels);
    if ((rc = check_overlap({{"out", out, all}},
                            {{"scores", out == scores ? nullptr : scores, all},   // (a thread reads what it then writes)
                             {"table", table, 4 * (int64_t)num_buckets * num_labels},
                             {"buckets", buckets, 4 * (int64_t)plan->n1}})) != CRF_OK ||
        (rc = check_device(plan)) != CRF_OK)
        return rc;
    const hipError_t e = crf::launch_width(plan->kp, plan->max_len, num_labels, table, buckets, num_buckets, scores, out,
                                           static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_width_bias launch");
}

int crf_biaffine_scores_biased(const crf_plan *plan, const uint16_t *rl, const uint16_t *rr, const uint16_t *w, int32_t d,
                               int32_t ldw, int32_t num_labels, const float *table, const int32_t *buckets,
                               int32_t num_buckets, float *scores, void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (rl == nullptr || rr == nullptr || w == nullptr || table == nullptr || buckets == nullptr || scores == nullptr)
        return fail(CRF_EINVAL, "rl/rr/w/table/buckets/scores is NULL");
    int rc = check_scorer(d, ldw, num_labels);
    if (rc != CRF_OK || (rc = check_buckets(num_buckets, num_labels)) != CRF_OK) return rc;
    if (misaligned(rl, 8) || misaligned(rr, 8) || misaligned(w, 8))
        return fail(CRF_EINVAL, "rl/rr/w must be 8-byte aligned");
    const int64_t rows = rows_bytes(plan, 2, d);
    if ((rc = check_overlap({{"scores", scores, scores_bytes(plan, num_labels)}},
                            {{"rl", rl, rows}, {"rr", rr, rows}, {"w", w, 2 * (int64_t)num_labels * d * ldw},
                             {"table", table, 4 * (int64_t)num_buckets * num_labels},
                             {"buckets", buckets, 4 * (int64_t)plan->n1}})) != CRF_OK ||
        (rc = check_device(plan)) != CRF_OK)
        return rc;
    static std::once_flag set[64];   // (see scorer_backward)
    std::call_once(set[plan->device & 63], [] {
        if (crf::set_biaffine_biased_attributes() != hipSuccess) (void)hipGetLastError();
    });
    const hipError_t e = crf::launch_biaffine_biased(plan->kp, rl, rr, w, d, ldw, num_labels, table, buckets, num_buckets,
                                                     scores, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_biaffine_scores_biased launch");
}

int crf_width_bias_bwd_workspace(const crf_plan *plan, int32_t num_labels, int64_t *bytes) {
    if (plan == nullptr || bytes == nullptr) return fail(CRF_EINVAL, "NULL argument");
    const int rc = check_buckets(1, num_labels);
    if (rc != CRF_OK) return rc;
    *bytes = crf::width_bwd_bytes(plan->kp, plan->max_len, num_labels);
    return ok();
}

int crf_width_bias_bwd(const crf_plan *plan, const float *grad_out, int32_t num_labels, const int32_t *buckets,
                       int32_t num_buckets, float *grad_scores, float *grad_table, void *workspace,
                       int64_t workspace_bytes, void *stream) {
    if (plan == nullptr) return fail(CRF_EINVAL, "plan is NULL");
    if (grad_out == nullptr || buckets == nullptr) return fail(CRF_EINVAL, "grad_out/buckets is NULL");
    int rc = check_buckets(num_buckets, num_labels);
    if (rc != CRF_OK) return rc;
    const int64_t all = scores_bytes(plan, num_labels), need = crf::width_bwd_bytes(plan->kp, plan->max_len, num_labels);
    if ((rc = check_workspace(workspace, workspace_bytes, need)) != CRF_OK ||
        (rc = check_overlap({{"grad_scores", grad_scores, all},
                             {"grad_table", grad_table, 4 * (int64_t)num_buckets * num_labels},
                             {"workspace", workspace, need}},
                            {{"grad_out", grad_out, all}, {"buckets", buckets, 4 * (int64_t)plan->n1}})) != CRF_OK ||
        (rc = check_device(plan)) != CRF_OK)
        return rc;
    if (grad_scores == nullptr && grad_table == nullptr) return ok();
    const hipError_t e = crf::launch_width_bwd(plan->kp, plan->max_len, num_labels, grad_out, buckets, num_buckets,
                                               grad_scores, grad_table, static_cast<char *>(workspace),
                                               static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_width_bias_bwd launch");
}

int crf_orthogonalize_workspace(int32_t count, int32_t rows, int32_t cols, int64_t *bytes) {
    if (bytes == nullptr) return fail(CRF_EINVAL, "NULL argument");
    const int rc = check_matrices(count, rows, cols, cols);
    if (rc != CRF_OK) return rc;
    *bytes = crf::ortho_bytes(count, rows, cols);
    return ok();
}

int crf_orthogonalize(const float *x, int32_t count, int32_t rows, int32_t cols, int32_t ld, const float *coefficients,
                      int32_t steps, float eps, float *out, void *workspace, int64_t workspace_bytes, void *stream) {
    if (x == nullptr || out == nullptr) return fail(CRF_EINVAL, "x/out is NULL");
    int rc = check_matrices(count, rows, cols, ld);
    if (rc != CRF_OK || (rc = check_coefficients(coefficients, steps, eps)) != CRF_OK) return rc;
    const int64_t all = 4 * (int64_t)count * rows * ld, need = crf::ortho_bytes(count, rows, cols);
    if ((rc = check_workspace(workspace, workspace_bytes, need)) != CRF_OK ||
        (rc = check_overlap({{"out", out, all}, {"workspace", workspace, need}}, {{"x", x, all}})) != CRF_OK ||
        (rc = set_update_attributes()) != CRF_OK)
        return rc;
    const hipError_t e = crf::launch_ortho(x, nullptr, nullptr, nullptr, out, count, rows, cols, ld, 0.f, false, 0.f, 0.f,
                                           eps, coefficients, steps, static_cast<char *>(workspace),
                                           static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_orthogonalize launch");
}

int crf_muon_step(const float *w, const float *grad, const float *momentum, int32_t count, int32_t rows, int32_t cols,
                  int32_t ld, float mu, int32_t nesterov, float rate, float decay, const float *coefficients, int32_t steps,
                  float eps, float *w_out, float *momentum_out, void *workspace, int64_t workspace_bytes, void *stream) {
    if (w == nullptr || grad == nullptr || momentum == nullptr || w_out == nullptr || momentum_out == nullptr)
        return fail(CRF_EINVAL, "w/grad/momentum/w_out/momentum_out is NULL");
    int rc = check_matrices(count, rows, cols, ld);
    if (rc != CRF_OK || (rc = check_coefficients(coefficients, steps, eps)) != CRF_OK) return rc;
    if (!finite_positive(mu)) return fail(CRF_EINVAL, "mu %g is negative or not finite", (double)mu);
    if (!finite_positive(rate)) return fail(CRF_EINVAL, "rate %g is negative or not finite", (double)rate);
    if (!finite_positive(decay) || decay > 1.f) return fail(CRF_EINVAL, "decay %g outside [0, 1]", (double)decay);
    const int64_t all = 4 * (int64_t)count * rows * ld, need = crf::ortho_bytes(count, rows, cols);
    // (in place: a thread reads what it then writes)
    if ((rc = check_workspace(workspace, workspace_bytes, need)) != CRF_OK ||
        (rc = check_overlap({{"w_out", w_out, all}, {"momentum_out", momentum_out, all}, {"workspace", workspace, need}},
                            {{"w", w == w_out ? nullptr : w, all}, {"grad", grad, all},
                             {"momentum", momentum == momentum_out ? nullptr : momentum, all}})) != CRF_OK ||
        (rc = set_update_attributes()) != CRF_OK)
        return rc;
    const hipError_t e = crf::launch_ortho(grad, momentum, w, momentum_out, w_out, count, rows, cols, ld, mu, nesterov != 0,
                                           1.f - decay, rate, eps, coefficients, steps, static_cast<char *>(workspace),
                                           static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, "crf_muon_step launch");
}

}  // extern "C"
