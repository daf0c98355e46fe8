/*
 * crf_inside.h -- C ABI of the MI355X (gfx950) batched tree-CRF library.
 *
 * Method: Zhang, Zhou & Li, "Fast and Accurate Neural CRF Constituency
 * Parsing" (IJCAI 2020).  For every sentence of a batch, given span scores
 * s(i,j), the library computes
 *   - log Z(x), the log partition function over all binary bracketings
 *     (Sec. 2.1, Eq. tree-prob), by the inside recursion of Sec. 3.1
 *     (Algorithm 1);
 *   - the span marginals p((i,j)|x) = d log Z / d s(i,j) (Sec. 3.2,
 *     Eq. partial-derivative), evaluated as exp(inside + outside - log Z)
 *     with the outside recursion run beside the inside one;
 *   - the 1-best tree argmax_y s(x,y) (Sec. 2.1, Eq. tree-argmax) by CKY,
 *     the same recursion with max in place of sum (Sec. 3.3);
 *   - for the one-stage labelled CRF (Sec. 4.2, Eq. tree-label-score),
 *     log Z, the per-label span marginals p((i,j,l)|x) and the best
 *     labelled tree;
 *   - MBR decoding over the marginals (Sec. 3.3), the gold-tree CRF loss
 *     and its gradient (Sec. 2.3, Eq. bracket-loss), and the labelling stage
 *     of the two-stage parser (Sec. 2.1, Eq. label-argmax);
 *   - the span (and label) scores themselves, from boundary representations
 *     by the biaffine scorer (Sec. 2.2, Eq. biaffine), and the scorer's
 *     backward pass, from the representations or from an 8-bit form of them;
 *   - log-probabilities of given trees and a clipped policy loss on them with
 *     its gradient, for training past the gold trees;
 *   - what else training a scorer takes: layer norm of the rows that it reads
 *     and a learned bias by a span's width, each with its gradients, and the
 *     update of its weights by their orthogonalised momentum.
 *
 * Conventions
 *   Fence posts.  A sentence of n words has boundaries 0..n; span (i,j),
 *   0 <= i < j <= n, covers words i..j-1 (the paper's inclusive (i, j-1)).
 *   Every legal tree contains all n width-1 spans and the root (0,n) and has
 *   2n-1 spans in all (Sec. 2.1; Fig. 1b); width-1 spans are scored.
 *
 *   Layout.  scores is float32, row-major [B][N1][N1] (unlabelled) or
 *   [B][N1][N1][L] (labelled), N1 = the padded side (>= max length + 1).
 *   s(i,j) of sentence b is scores[(b*N1 + i)*N1 + j] (times L, plus l, when
 *   labelled).  Only cells 0 <= i < j <= n_b are read; every other cell may
 *   hold anything, NaN included.  marginals has the layout of scores and only
 *   its valid cells are written: the rest of the buffer is left untouched.
 *   Outputs are in the caller's sentence order.
 *
 *   Memory.  Every float/int pointer passed to a compute call is device memory
 *   owned by the caller; the library never frees it.  lengths_host in
 *   crf_plan_create is host memory, read only during the call.  The plan owns
 *   its device copies of the lengths and schedule, a workspace for
 *   sentences whose chart does not fit in LDS and, with such sentences, a
 *   257 KB area for the teams below; they are allocated by crf_plan_create
 *   and freed by crf_plan_destroy.  Compute calls allocate nothing.
 *
 *   Teams.  When a call has only a few workspace sentences, each pass may run
 *   on a team of 8 or 16 workgroups of one XCD that wait for each other at
 *   every width step: unlabelled plans with at most 16 workspace sentences of
 *   which one has more than 450 words, and calls of labelled plans with at
 *   most 32 workspace sentence passes in one launch.
 *   Such a launch waits until all its workgroups are resident at once (it
 *   is sized to fit an otherwise idle device); work from other streams
 *   delays it.  A wait that lasts about 2^21 polls (a second or two) ends
 *   the launch, and the outputs of its workspace sentences are invalid: log
 *   Z and best score NaN when a width step's wait ran out, left unwritten
 *   when the launch's workgroups never were resident together (the
 *   log-probabilities and log Z of crf_tree_logprobs, and the loss,
 *   log-probabilities and gradient of crf_policy_loss, are NaN in either
 *   case; marginals and other gradients do not tell).  Two plans' team
 *   launches running at once on different streams
 *   can hold each other's room that way: issue calls that may form teams on
 *   one stream, or create the plans with CRF_NO_TEAMS.  Results are
 *   bit-identical to those of one workgroup per pass.
 *
 *   Streams.  `stream` is a hipStream_t (NULL = the null stream).  Compute
 *   calls only enqueue work and never synchronise.  Calls on one plan must
 *   not overlap on the device: issue them on one stream, or order them with
 *   events.  A plan owns device state that its calls use while they run --
 *   the workspace that holds the charts
 *   and CKY split tables of sentences too long for LDS (crf_plan_info:
 *   workspace_users) and the team area -- and two overlapping calls would
 *   share it.  Different
 *   plans share nothing and may run concurrently on any streams (but see
 *   Teams below for calls with a few workspace sentences).
 *
 *   Errors.  Every call returns a status (CRF_OK = 0).  Arguments are checked
 *   on the host before any HIP call is made, so a rejected call has no effect
 *   on the device.  crf_last_error() gives a message for the last failure on
 *   the calling thread.  Scores must be finite inside the valid region; NaN
 *   or infinities there give unspecified (but memory-safe) results.
 */
#ifndef CRF_INSIDE_H
#define CRF_INSIDE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    CRF_OK = 0,
    CRF_EINVAL = 1,        /* bad argument: null pointer, size or length out of range */
    CRF_ENOMEM = 2,        /* host or device allocation failed (crf_plan_create only) */
    CRF_EHIP = 3,          /* HIP runtime or launch error (see crf_last_error) */
    CRF_EUNSUPPORTED = 4   /* valid but not implemented, e.g. decode of labelled scores */
};

#define CRF_MAX_LEN 1023      /* longest sentence, in words */
#define CRF_MAX_LABELS 4096   /* most labels per span */
#define CRF_MAX_TREES 64      /* most candidate trees per sentence */
#define CRF_MAX_ROW 8192      /* longest activation row held in 8 bits */
#define CRF_MAX_BUCKETS 1024  /* most buckets of span widths */
#define CRF_MAX_STEPS 32      /* most Newton-Schulz steps */

/* Types of rows that a call takes in more than one. */
#define CRF_BF16 0            /* bf16 bit patterns */
#define CRF_F32 1             /* float32 */

/* Plan flags. */
#define CRF_FORCE_SPILL 0x1u  /* run every sentence on the workspace-chart kernels */
#define CRF_NO_TEAMS 0x2u     /* one workgroup per workspace sentence pass, never teams */

typedef struct crf_plan crf_plan;

typedef struct {
    int32_t batch;           /* B */
    int32_t n1;              /* padded side N1 */
    int32_t num_labels;      /* L (1 = unlabelled) */
    int32_t max_len;         /* longest sentence */
    int32_t lds_count;       /* sentences whose inside chart lives in LDS */
    int32_t spill_count;     /* sentences whose inside chart lives in the workspace */
    int64_t workspace_bytes; /* device workspace owned by the plan */
    int32_t lds_bytes_inside;/* dynamic LDS per workgroup, inside kernels (the
                                sentences whose chart lives in LDS) */
    int32_t lds_bytes_cky;   /* dynamic LDS per workgroup, CKY kernel */
    int32_t cky_spill_count; /* sentences whose CKY chart lives in the workspace */
    int32_t split_ws_count;  /* sentences whose CKY chart is in LDS but whose
                                split table is in the workspace */
    int32_t workspace_users; /* sentences that use the workspace in some call
                                (any of the three above) */
    int32_t fused_queue;     /* 0: no launch pulls work from a counter of the
                                plan's any more */
    int32_t mbr_fused;       /* 1 if crf_mbr_decode runs the sentences whose
                                charts live in LDS in one launch (0: none do) */
} crf_plan_stats;

/*
 * crf_plan_create -- validate a batch shape and build its schedule.
 *   out          receives the plan (set to NULL on failure).
 *   lengths_host host int32[batch]: sentence lengths n_b, 1 <= n_b <= n1-1.
 *   batch        B >= 1.
 *   n1           padded side of the score block, 2 <= n1 <= CRF_MAX_LEN+1.
 *   num_labels   L, 1 <= L <= CRF_MAX_LABELS; 1 = unlabelled scores.
 *   flags        0, or CRF_FORCE_SPILL and/or CRF_NO_TEAMS.
 * Uses the current HIP device; later calls must run with that device current.
 * Returns CRF_EINVAL (nothing allocated), CRF_ENOMEM or CRF_EHIP.
 */
int crf_plan_create(crf_plan **out, const int32_t *lengths_host, int32_t batch, int32_t n1,
                    int32_t num_labels, uint32_t flags);

/* Free a plan and its device memory (NULL is accepted).  Synchronises the
 * device first so that no enqueued call still uses it. */
int crf_plan_destroy(crf_plan *plan);

/* Sizes and schedule summary of a plan (host only, no HIP call). */
int crf_plan_info(const crf_plan *plan, crf_plan_stats *out);

/*
 * crf_inside_fwd -- log partition function (Sec. 2.1, Eq. tree-prob; Sec. 3.1,
 * Algorithm 1).
 *   scores  device float32, layout above.
 *   logZ    device float32[B]: log Z(x_b).
 */
int crf_inside_fwd(const crf_plan *plan, const float *scores, float *logZ, void *stream);

/*
 * crf_inside_bwd -- span marginals as the gradient of log Z (Sec. 3.2,
 * Eq. partial-derivative).  The inside chart is recomputed on chip.
 *   grad_logZ  device float32[B] upstream gradient, or NULL for all ones.
 *   marginals  device float32, layout of scores: grad_logZ[b] * p((i,j)|x_b)
 *              (labelled: grad_logZ[b] * p((i,j,l)|x_b)) on valid cells only.
 */
int crf_inside_bwd(const crf_plan *plan, const float *scores, const float *grad_logZ,
                   float *marginals, void *stream);

/* crf_inside_fwd_bwd -- both of the above in one pass over the chart.
 * logZ may be NULL. */
int crf_inside_fwd_bwd(const crf_plan *plan, const float *scores, const float *grad_logZ,
                       float *logZ, float *marginals, void *stream);

/*
 * crf_cky_decode -- 1-best unlabelled tree (Sec. 2.1, Eq. tree-argmax) by CKY
 * (Sec. 3.3).  The chart is float64: beta(i,i+1) = s(i,i+1),
 * beta(i,j) = (max_k (beta(i,k) + beta(k,j))) + s(i,j); among equal maxima
 * the lowest split k is kept.
 *   spans  device int32[B][2*(N1-1)-1][2]: the 2n_b-1 spans (i,j) of the tree
 *          in preorder (i ascending, then j descending), then rows of -1.
 *   best   device float32[B] score of that tree, or NULL.
 * Unlabelled plans only (CRF_EUNSUPPORTED otherwise).
 */
int crf_cky_decode(const crf_plan *plan, const float *scores, int32_t *spans, float *best,
                   void *stream);

/*
 * crf_inside_fwd_bwd_cky -- crf_inside_fwd_bwd and crf_cky_decode in one
 * launch, their workgroups interleaved so the two run concurrently.  Same
 * arguments and results as the two calls (logZ and best may be NULL).
 * Unlabelled plans only (CRF_EUNSUPPORTED otherwise).
 */
int crf_inside_fwd_bwd_cky(const crf_plan *plan, const float *scores, const float *grad_logZ,
                           float *logZ, float *marginals, int32_t *spans, float *best,
                           void *stream);

/*
 * crf_mbr_decode -- MBR decoding (Sec. 3.3, "Decoding"): the CKY tree with the
 * span marginals p((i,j)|x) in place of the span scores in Eq. tree-score and
 * Eq. tree-argmax, i.e. the tree whose spans' marginals sum highest.  One
 * pass: the inside and outside sweeps write the marginals, and the same
 * workgroup then runs CKY over them (float64 chart, lowest split on ties, as
 * crf_cky_decode) while its bundle is still on chip.
 *   logZ       device float32[B] or NULL: log Z(x_b).
 *   marginals  device float32, layout of scores (required, must not alias
 *              scores): p((i,j)|x_b) on valid cells; the trees are decoded
 *              from exactly these float32 values.
 *   spans      device int32[B][2*(N1-1)-1][2], as crf_cky_decode.
 *   best       device float32[B] or NULL: the sum of the marginals over the
 *              tree (float64 chart, rounded).
 * Unlabelled plans only (CRF_EUNSUPPORTED otherwise).
 */
int crf_mbr_decode(const crf_plan *plan, const float *scores, float *logZ, float *marginals, int32_t *spans,
                   float *best, void *stream);

/*
 * crf_gold_loss -- the sentence-level CRF loss of a gold tree (Sec. 2.3,
 * Eq. bracket-loss), L = log Z(x) - s(x,y), with s(x,y) the sum of the gold
 * spans' scores (Eq. tree-score), and its gradient with respect to the scores,
 * dL/ds(i,j) = p((i,j)|x) - 1[(i,j) in y] (the marginals of Sec. 3.2 minus
 * the gold indicator).
 *   gold_spans  device int32[B][2*(N1-1)-1][2]: the first 2n_b-1 rows of
 *               sentence b are its gold tree's spans (i,j) (the layout
 *               crf_cky_decode writes; any order).  Rows that are not spans
 *               of the sentence (0 <= i < j <= n_b) are skipped; a repeated
 *               span adds its score to s(x,y) again but 1 to the indicator.
 *   grad_loss   device float32[B] upstream gradient dOut/dL, or NULL for 1.
 *   loss        device float32[B]: L (not scaled by grad_loss).
 *   grad_scores device float32, layout of scores (must not alias scores):
 *               grad_loss[b] * (p((i,j)|x_b) - 1[(i,j) in y_b]) on valid cells
 *               only.
 * Unlabelled plans only (CRF_EUNSUPPORTED otherwise).
 */
int crf_gold_loss(const crf_plan *plan, const float *scores, const int32_t *gold_spans, const float *grad_loss,
                  float *loss, float *grad_scores, void *stream);

/*
 * crf_cky_decode_labeled -- one-stage labelled decoding (Sec. 4.2,
 * Eq. tree-label-score; Sec. 2.1, time-complexity paragraph): the labelled
 * tree maximising the sum of s(i,j,l) over its labelled spans.  Each span's
 * label is free, so this is CKY (as crf_cky_decode) over the float32 maxima
 * max_l s(i,j,l), each of the tree's spans labelled with the lowest label
 * attaining its maximum.
 *   scores  device float32 [B][N1][N1][L], L = the plan's num_labels.
 *   spans   device int32[B][2*(N1-1)-1][2], as crf_cky_decode.
 *   labels  device int32[B][2*(N1-1)-1]: the label of each span row, -1 on
 *           the rows past the tree.
 *   best    device float32[B] or NULL: the labelled tree's score.
 */
int crf_cky_decode_labeled(const crf_plan *plan, const float *scores, int32_t *spans, int32_t *labels, float *best,
                           void *stream);

/*
 * crf_label_spans -- the labelling stage of the two-stage parser (Sec. 2.1,
 * Eq. label-argmax): every span (i,j) of a given tree independently takes
 * argmax_l s(i,j,l) (the lowest such label on ties).
 *   label_scores  device float32 [B][N1][N1][num_labels] (N1 and B of the
 *                 plan; the plan's own num_labels is not used).
 *   num_labels    1 <= num_labels <= CRF_MAX_LABELS.
 *   spans         device int32[B][2*(N1-1)-1][2], e.g. crf_cky_decode's or
 *                 crf_mbr_decode's output.
 *   labels        device int32[B][2*(N1-1)-1]: the label of every row that is
 *                 a span of its sentence (0 <= i < j <= n_b), else -1.
 */
int crf_label_spans(const crf_plan *plan, const float *label_scores, int32_t num_labels, const int32_t *spans,
                    int32_t *labels, void *stream);

/*
 * crf_biaffine_scores -- the biaffine span scorer that produces the span
 * scores (Sec. 2.2, Eq. biaffine): s(i,j) = [r^l_i ; 1]^T W r^r_j from the
 * left boundary representation of fence post i and the right one of fence
 * post j, W of (d+1) x d entries (the appended 1 makes its last row a bias on
 * r^r_j); one W per label for label scores (Sec. 2.2, label scoring):
 * s(i,j,l) = [r^l_i ; 1]^T W_l r^r_j.  bf16 inputs, fp32 products and sums
 * on the matrix cores (MFMA); the inner (d x d) product stays on chip.
 *   rl, rr      device bf16 bit patterns [B][N1][d]: r^l_i and r^r_i of
 *               sentence b at [(b*N1 + i)*d]; rows past n_b are not read.
 *               8-byte aligned.
 *   w           device bf16 bit patterns [num_labels][d][ldw], W transposed:
 *               w[(l*d + c)*ldw + a] = W_l[a][c] for a <= d (a = d is the bias
 *               row); entries a > d are not read.  8-byte aligned.
 *   d           4 <= d <= 508, a multiple of 4 (the paper's d is 500, and
 *               100 for the label scorer).
 *   ldw         row stride of w, >= d+1 and a multiple of 4.
 *   num_labels  number of W (1 for span scores).
 *   scores      device float32, [B][N1][N1] when num_labels = 1 (the layout
 *               the CRF calls take), else [B][N1][N1][num_labels]; only cells
 *               0 <= i < j <= n_b are written.
 * B, N1 and the lengths are the plan's (its own num_labels is not used).
 */
int crf_biaffine_scores(const crf_plan *plan, const uint16_t *rl, const uint16_t *rr, const uint16_t *w,
                        int32_t d, int32_t ldw, int32_t num_labels, float *scores, void *stream);

/*
 * crf_inside_fwd_bwd_cky_noalloc -- crf_inside_fwd_bwd_cky for callers that
 * cannot allocate device memory or must not touch the plan's device state
 * while they run (code under HIP graph capture, tight serving loops,
 * harnesses that forbid allocation).  Same arguments and results as
 * crf_inside_fwd_bwd_cky; the plan's workspace is not used: the call takes
 * one (and a work counter) from a static scratch array of the library,
 * 8 MiB per GPU, held from the library's first use on a device until the
 * process ends.  It calls no allocation routine; it enqueues a small kernel
 * that clears the array's counter, then the launches of the fused call
 * (with one workgroup per workspace sentence pass: no teams).
 *   Returns CRF_EINVAL when the plan needs more workspace than the array
 *   holds (8 MiB less 256 bytes), e.g. a batch with many sentences longer
 *   than 141 words.  The need counted is that of the charts of single spans,
 *   which can be less than crf_plan_info's workspace_bytes (that also covers
 *   the charts in tiles of spans); a plan whose tile charts do not fit the
 *   array runs on the charts of single spans.
 *   Every such call on one GPU shares that GPU's array, whatever the plan:
 *   calls of this entry point that overlap on one GPU race (issue them on
 *   one stream, or order them with events).
 */
int crf_inside_fwd_bwd_cky_noalloc(const crf_plan *plan, const float *scores, const float *grad_logZ,
                                   float *logZ, float *marginals, int32_t *spans, float *best,
                                   void *stream);

/*
 * Workspaces.  The calls below that take one use it, device memory of the
 * caller of at least the size that the plan's query gives, 256-byte aligned,
 * only while they run: calls that may overlap need one each (two graphs that
 * are replayed side by side too).  The tree calls still use the plan's own
 * workspace like the others, so they must not overlap other calls on the plan;
 * packing, unpacking, the scorer's backward pass, layer norm and the width bias
 * use nothing of it and may.
 * In all of them no output, and not the workspace, may overlap an input or
 * another output (CRF_EINVAL, by the arrays' full sizes).
 */

/* crf_tree_workspace -- bytes of workspace of crf_tree_logprobs and
 * crf_policy_loss. */
int crf_tree_workspace(const crf_plan *plan, int64_t *bytes);

/*
 * crf_tree_logprobs -- log-probabilities of given trees (Sec. 2.1,
 * Eq. tree-prob): log p(y|x) = s(x,y) - log Z(x), s(x,y) the sum of the
 * spans' scores (Eq. tree-score); sums and differences in float64.
 *   trees       device int32 [B][num_trees][2*(N1-1)-1][2], 8-byte aligned: of
 *               each tree the first 2n_b-1 rows are its spans (i,j) (what
 *               crf_cky_decode writes; any order).  Rows that are not spans of
 *               the sentence (0 <= i < j <= n_b) are skipped; a repeated span
 *               adds its score again.
 *   num_trees   G, 1 <= G <= CRF_MAX_TREES.
 *   counts      device int32[B]: the first counts[b] trees of sentence b are
 *               there (clamped to 0..G), or NULL: all of them.
 *   logp        device float32 [B][G]: log p of the trees that are there; the
 *               others' entries are left as they were.
 *   logZ        device float32 [B], or NULL: log Z(x_b).
 * Unlabelled plans only (CRF_EUNSUPPORTED otherwise).
 */
int crf_tree_logprobs(const crf_plan *plan, const float *scores, const int32_t *trees, int32_t num_trees,
                      const int32_t *counts, float *logp, float *logZ, void *workspace, int64_t workspace_bytes,
                      void *stream);

/*
 * crf_tree_logprobs_bwd -- the gradient of sum_g u_g log p(y_g|x_b) with
 * respect to the scores, u = grad_logp:
 *   sum_{g: (i,j) in y_g} u_g - (sum_g u_g) p((i,j)|x_b).
 *   trees, num_trees, counts: as crf_tree_logprobs; a repeated span counts
 *               once.
 *   grad_logp   device float32 [B][G]; the entries of trees that are not there
 *               are not read.
 *   grad_scores device float32, layout of scores (must not alias scores):
 *               valid cells only.
 * Unlabelled plans only (CRF_EUNSUPPORTED otherwise).  Needs no workspace.
 */
int crf_tree_logprobs_bwd(const crf_plan *plan, const float *scores, const int32_t *trees, int32_t num_trees,
                          const int32_t *counts, const float *grad_logp, float *grad_scores, void *stream);

/*
 * crf_policy_loss -- clipped policy loss of each sentence's trees with a KL
 * term, and its gradient with respect to the scores.  With A the advantages,
 * r_g = exp(log p_g - old_g), q_g = ref_g - log p_g and c = counts[b]:
 *   L_b = 1/c sum_g [ -min(r_g A_g, clip(r_g, 1 - clip_low, 1 + clip_high) A_g)
 *                     + kl_coef (exp(q_g) - q_g - 1) ],
 *   dL_b/ds(i,j) = sum_{g: (i,j) in y_g} c_g - (sum_g c_g) p((i,j)|x_b),
 *   c_g = dL_b/dlog p_g = 1/c [ -r_g A_g [r_g A_g <= clip(r_g) A_g]
 *                               + kl_coef (1 - exp(q_g)) ].
 * log p_g - old_g and q_g above 80 are taken as 80.  A sentence without trees
 * has the loss 0 and the gradient 0; one with a NaN among its trees'
 * advantages, old_logp or ref_logp has the loss NaN and a gradient of NaN.
 *   trees, num_trees, counts, logp (or NULL): as crf_tree_logprobs; a repeated
 *               span counts once in the gradient.
 *   advantages, old_logp  device float32 [B][G].
 *   ref_logp    device float32 [B][G], or NULL: no KL term (kl_coef is 0, and
 *               then it is not read).
 *   clip_low    0 <= clip_low <= 1; clip_high >= 0; kl_coef >= 0.
 *   grad_loss   device float32[B] upstream gradient dOut/dL_b, or NULL for 1.
 *   loss        device float32[B]: L_b (not scaled by grad_loss).  loss and logp
 *               must not alias an input.
 *   grad_scores device float32, layout of scores (must not alias scores):
 *               grad_loss[b] dL_b/ds(i,j) on valid cells only.
 * Unlabelled plans only (CRF_EUNSUPPORTED otherwise).
 */
int crf_policy_loss(const crf_plan *plan, const float *scores, const int32_t *trees, int32_t num_trees,
                    const int32_t *counts, const float *advantages, const float *old_logp, const float *ref_logp,
                    float clip_low, float clip_high, float kl_coef, const float *grad_loss, float *loss, float *logp,
                    float *grad_scores, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * crf_pack_rows -- activation rows in 8 bits, for what a backward pass keeps.
 * Blocks of 32 entries of a row share a power of two: with m the largest
 * finite magnitude of a block, code = e4m3(x 2^-s) (nearest, ties to even),
 * s = max(ceil(log2(m / 448)), -127), and the code stands for code 2^s.
 * Magnitudes from 1.9375 2^127 up are held as 1.875 2^127 (the nearest code
 * would stand for 2^128).  Infinities and NaN become the code's NaN.
 *   x       device bf16 bit patterns [B][N1][d], 8-byte aligned; rows past n_b
 *           are not read.
 *   d       4 <= d <= CRF_MAX_ROW, a multiple of 4.
 *   codes   device uint8 [B][N1][dc], dc = d rounded up to a multiple of 32,
 *           16-byte aligned: e4m3 (no infinities) bit patterns, zeros past d.
 *   scales  device uint8 [B][N1][dc/32]: s + 127.
 * Rows past n_b are left as they were.  x and codes must not alias.  B, N1 and
 * the lengths are the plan's.
 */
int crf_pack_rows(const crf_plan *plan, const uint16_t *x, int32_t d, uint8_t *codes, uint8_t *scales, void *stream);

/* crf_unpack_rows -- the values that packed rows stand for, as bf16 (exact but
 * for values below 2^-126); rows past n_b are left as they were. */
int crf_unpack_rows(const crf_plan *plan, const uint8_t *codes, const uint8_t *scales, int32_t d, uint16_t *x,
                    void *stream);

/* crf_biaffine_bwd_workspace -- bytes of workspace of crf_biaffine_bwd and
 * crf_biaffine_bwd_packed for representations of d dimensions and num_labels
 * labels. */
int crf_biaffine_bwd_workspace(const crf_plan *plan, int32_t d, int32_t num_labels, int64_t *bytes);

/*
 * crf_biaffine_bwd -- the backward pass of crf_biaffine_scores (Sec. 2.2,
 * Eq. biaffine).  With G_l(i,j) = dL/ds(i,j,l) on 0 <= i < j <= n_b,
 *   dL/dr^l_i = sum_l sum_j G_l(i,j) W_l r^r_j  (W_l's first d rows),
 *   dL/dr^r_j = sum_l sum_i G_l(i,j) W_l^T [r^l_i ; 1],
 *   dL/dW_l   = sum_b sum_{i<j} G_l(i,j) [r^l_i ; 1] r^r_j^T.
 * Products on the matrix cores with fp32 sums; G_l and the inner one of two
 * products enter as two bf16 parts (2^-16 of each is lost at most).
 *   rl, rr, w, d, ldw, num_labels: as crf_biaffine_scores.
 *   grad_scores device float32, the layout of the scores; only cells
 *               0 <= i < j <= n_b are read.
 *   grad_rl, grad_rr  device bf16 bit patterns [B][N1][d], 8-byte aligned, or
 *               NULL: rows 0..n_b are written.
 *   grad_w      device float32 [num_labels][d][ldw], 16-byte aligned, or NULL:
 *               the layout of w; entries a <= d are written.
 * Sums run in a fixed order: equal calls give equal bits.  An infinity or NaN
 * among a sentence's representations or its spans' gradients makes rows of its
 * own grad_rl and grad_rr NaN (short sentences: all rows of the one that the
 * representation enters) and shows in grad_w; other sentences' rows are as
 * without it.  W must be finite.  No gradient may alias an input or another one.
 */
int crf_biaffine_bwd(const crf_plan *plan, const uint16_t *rl, const uint16_t *rr, const uint16_t *w, int32_t d,
                     int32_t ldw, int32_t num_labels, const float *grad_scores, uint16_t *grad_rl, uint16_t *grad_rr,
                     float *grad_w, void *workspace, int64_t workspace_bytes, void *stream);

/* crf_biaffine_bwd_packed -- the same from representations in the 8-bit form
 * of crf_pack_rows (the gradients are those at the values that the codes stand
 * for). */
int crf_biaffine_bwd_packed(const crf_plan *plan, const uint8_t *rl_codes, const uint8_t *rl_scales,
                            const uint8_t *rr_codes, const uint8_t *rr_scales, const uint16_t *w, int32_t d, int32_t ldw,
                            int32_t num_labels, const float *grad_scores, uint16_t *grad_rl, uint16_t *grad_rr,
                            float *grad_w, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * crf_layer_norm -- layer norm of activation rows: with m and v the mean and the
 * variance of a row's d entries,
 *   y = (x - m) / sqrt(v + eps) * gamma + beta.
 * Sums in float32; the variance is that of the deviations from the mean, and what
 * the mean's rounding leaves in them is taken off.
 *   x       device [B][N1][d], bf16 bit patterns (x_type CRF_BF16, 8-byte
 *           aligned) or float32 (CRF_F32); rows past n_b are not read.
 *   d       4 <= d <= CRF_MAX_ROW, a multiple of 4.
 *   gamma, beta  device float32[d], or NULL: 1 and 0.
 *   eps     finite, 2^-126 (float32's least normal number) or more.
 *   y       device bf16 bit patterns [B][N1][d], 8-byte aligned; must not alias x.
 * A row with an infinity or NaN, or whose sum of squared deviations passes what
 * float32 holds, becomes NaN, as may one of entries past 2^76 in size, whose mean's
 * rounding or sum can do so; other rows are as without it.  Rows past n_b are left
 * as they were.  B, N1 and the lengths are the plan's.
 */
int crf_layer_norm(const crf_plan *plan, const void *x, int32_t x_type, int32_t d, const float *gamma, const float *beta,
                   float eps, uint16_t *y, void *stream);

/* crf_layer_norm_bwd_workspace -- bytes of workspace of crf_layer_norm_bwd. */
int crf_layer_norm_bwd_workspace(const crf_plan *plan, int32_t d, int64_t *bytes);

/*
 * crf_layer_norm_bwd -- the backward pass of crf_layer_norm.  With h the
 * normalised row, r = 1 / sqrt(v + eps) and u = grad_y gamma,
 *   grad_x = r (u - mean(u) - h mean(u h)),
 *   grad_gamma = sum of grad_y h over the batch's rows, grad_beta = sum of grad_y.
 * The statistics are taken from x again.
 *   x, x_type, d, gamma, eps: as crf_layer_norm.
 *   grad_y      device bf16 bit patterns [B][N1][d], 8-byte aligned; rows past
 *               n_b are not read.
 *   grad_x      device, x's type and layout, or NULL: rows 0..n_b are written.
 *   grad_gamma, grad_beta  device float32[d], or NULL.
 * Sums run in a fixed order: equal calls give equal bits.
 */
int crf_layer_norm_bwd(const crf_plan *plan, const void *x, int32_t x_type, int32_t d, const float *gamma,
                       const uint16_t *grad_y, float eps, void *grad_x, float *grad_gamma, float *grad_beta,
                       void *workspace, int64_t workspace_bytes, void *stream);

/*
 * crf_width_bias -- a learned bias by a span's width, widths in buckets:
 *   out(i,j,l) = scores(i,j,l) + table[buckets[j - i]][l].
 *   scores      device float32, [B][N1][N1] when num_labels = 1, else
 *               [B][N1][N1][num_labels]; only cells 0 <= i < j <= n_b are read.
 *   num_labels  1 <= num_labels <= CRF_MAX_LABELS (the plan's own is not used).
 *   table       device float32 [num_buckets][num_labels].
 *   buckets     device int32[N1]: the bucket of each width (entry 0 is not
 *               read); spans whose bucket is outside 0 .. num_buckets - 1 get
 *               no bias.
 *   num_buckets 1 <= num_buckets <= CRF_MAX_BUCKETS.
 *   out         device float32, layout of scores, valid cells only; may be
 *               scores itself, must not overlap it otherwise.
 */
int crf_width_bias(const crf_plan *plan, const float *scores, int32_t num_labels, const float *table,
                   const int32_t *buckets, int32_t num_buckets, float *out, void *stream);

/*
 * crf_biaffine_scores_biased -- crf_biaffine_scores and crf_width_bias in one:
 * the same scores, the bias added to each (in float32) where it is written.
 * scores must not overlap an input.
 */
int crf_biaffine_scores_biased(const crf_plan *plan, const uint16_t *rl, const uint16_t *rr, const uint16_t *w, int32_t d,
                               int32_t ldw, int32_t num_labels, const float *table, const int32_t *buckets,
                               int32_t num_buckets, float *scores, void *stream);

/* crf_width_bias_bwd_workspace -- bytes of workspace of crf_width_bias_bwd. */
int crf_width_bias_bwd_workspace(const crf_plan *plan, int32_t num_labels, int64_t *bytes);

/*
 * crf_width_bias_bwd -- the backward pass of crf_width_bias.
 *   grad_out    device float32, layout of the scores; valid cells are read.
 *   grad_scores device float32, the same layout, or NULL: grad_out on valid
 *               cells (the others are left as they were); must not alias it.
 *   grad_table  device float32 [num_buckets][num_labels], or NULL: for each
 *               bucket and label the sum of grad_out over the batch's spans of
 *               the bucket's widths (0 where it has none).
 * Sums in float32 in a fixed order: equal calls give equal bits.
 */
int crf_width_bias_bwd(const crf_plan *plan, const float *grad_out, int32_t num_labels, const int32_t *buckets,
                       int32_t num_buckets, float *grad_scores, float *grad_table, void *workspace,
                       int64_t workspace_bytes, void *stream);

/* crf_orthogonalize_workspace -- bytes of workspace of crf_orthogonalize and
 * crf_muon_step.  The three calls take no plan and run on the current device. */
int crf_orthogonalize_workspace(int32_t count, int32_t rows, int32_t cols, int64_t *bytes);

/*
 * crf_orthogonalize -- matrices with their singular values brought towards 1 by
 * Newton-Schulz products: X = x / (|x|_F + eps), then for each step's (a, b, c)
 *   A = X X^T,  X <- a X + (b A + c A A) X.
 * Operands of the products are held as two float16 parts (22 bits; float32 where
 * the shorter side is at most 16 and the longer at most 2,048), sums are float32;
 * |x|_F is summed in float64.
 *   x, out        device float32 [count][rows][ld], entries [..][cols] of a row;
 *                 the others are neither read nor written.  out must not alias x.
 *   count         1 <= count <= CRF_MAX_LABELS.
 *   rows, cols    1 to CRF_MAX_ROW each; ld >= cols.
 *   coefficients  host float[steps][3], read during the call.  Singular values
 *                 from [0, 1] must stay in [0, 4] after every step, and
 *                 |a + b s^2 + c s^4| within 60 (CRF_EINVAL otherwise: the parts
 *                 of larger values would overflow); none past 1,000 in size.
 *   steps         1 <= steps <= CRF_MAX_STEPS.
 *   eps           positive.  The parts of x / (|x|_F + eps) are whole multiples of
 *                 2^-36, so where |x|_F is far below eps they have few digits.
 * A matrix with an infinity or NaN gives NaN everywhere, the others are as
 * without it; a matrix of zeros gives zeros.
 */
int crf_orthogonalize(const float *x, int32_t count, int32_t rows, int32_t cols, int32_t ld, const float *coefficients,
                      int32_t steps, float eps, float *out, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * crf_muon_step -- weights moved by their orthogonalised momentum: with X the
 * result of crf_orthogonalize for U,
 *   momentum_out = mu momentum + grad,
 *   U = grad + mu momentum_out (nesterov), or momentum_out,
 *   w_out = (1 - decay) w - rate X.
 *   w, grad, momentum, w_out, momentum_out  device float32 [count][rows][ld] (the
 *               scorer's W as it lies: rows d, cols d + 1).  w_out may be w and
 *               momentum_out momentum; no other buffers may overlap.
 *   mu, rate    at least 0; 0 <= decay <= 1.
 */
int crf_muon_step(const float *w, const float *grad, const float *momentum, int32_t count, int32_t rows, int32_t cols,
                  int32_t ld, float mu, int32_t nesterov, float rate, float decay, const float *coefficients, int32_t steps,
                  float eps, float *w_out, float *momentum_out, void *workspace, int64_t workspace_bytes, void *stream);

/* Static description of a status code. */
const char *crf_status_string(int status);

/* Message for the last failing call on this thread ("" if none). */
const char *crf_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* CRF_INSIDE_H */
