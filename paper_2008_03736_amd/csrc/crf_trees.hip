// crf_trees.hip -- log-probabilities of given trees and the clipped policy
// loss on them.
//
// A tree y of a sentence x has the probability p(y|x) = exp(s(x,y)) / Z(x)
// (Sec. 2.1, Eq. tree-prob), so log p = s(x,y) - log Z, with s(x,y) the sum of
// its spans' scores.  A sentence's G candidate trees with advantages A_g, the
// log-probabilities old_g under the policy that drew them and ref_g under a
// reference have the loss
//     L = 1/c sum_g -min(r_g A_g, clip(r_g, 1 - lo, 1 + hi) A_g) + beta k_g,
//     r_g = exp(log p_g - old_g),  k_g = exp(q_g) - q_g - 1,  q_g = ref_g - log p_g
// over its c candidates, whose gradient by log p_g is
//     c_g = 1/c (-A_g r_g [where the first of the two is the smaller] + beta (1 - exp(q_g))),
// and d log p_g / d s(i,j) = 1[(i,j) in y_g] - p((i,j)|x), so that
//     dL/ds(i,j) = sum_{g: (i,j) in y_g} c_g - (sum_g c_g) p((i,j)|x).
//
// Two launches: the inside sweep (with the marginals for the loss, which it
// leaves in the gradient's buffer), then the kernel below, a workgroup per
// sentence, or per stripe of at most kTreeCells cells of a long sentence's rows
// (KernelPlan::tree_recs; each sums the trees anew, which for its few
// workgroups is cheaper than another launch).
//
// The second pass is bound by its chain of memory round trips (rows of the
// trees, their scores, the cells), so what does not depend on them is loaded
// first, and stripes are kept small (8 KB of masks) so that eight workgroups
// share a CU: 4 trees of 5,000 sentences 52.6 us with stripes of 8,192 cells
// and nothing loaded ahead.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "crf_internal.h"

namespace crf {
namespace {

constexpr int kTreeThreads = 256;
constexpr int kAhead = 4;   // rows of a tree, and cells of the gradient, that a lane has in flight

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) v += __shfl_xor(v, k, 64);
    return v;
}

// NaN, by the bits: the build takes no account of it in comparisons, and a
// minimum drops it.  (The compiler knows this test of a float's bits, and that
// it may take it for false: the asm hides that they are a float's.)
__device__ __forceinline__ bool is_nan(uint32_t u) {
    asm("" : "+v"(u));
    return (u & 0x7FFFFFFFu) > 0x7F800000u;
}
__device__ __forceinline__ bool is_nan(uint64_t u) {
    asm("" : "+v"(u));
    return (u & 0x7FFFFFFFFFFFFFFFull) > 0x7FF0000000000000ull;
}
__device__ __forceinline__ float or_nan(bool lost, float x) {
    uint32_t u = lost ? 0x7FC00000u : __builtin_bit_cast(uint32_t, x);
    asm("" : "+v"(u));
    return __builtin_bit_cast(float, u);
}

// What a launch is for: log p alone, the gradient of given weights of log p,
// or the policy loss and its gradient.
enum TreeMode { kTreeLogp, kTreeBack, kTreePolicy };

struct PolicyArgs {
    const float *grad_logp;   // kTreeBack: [B][G]
    const float *adv, *old_logp, *ref_logp, *grad_loss;
    float clip_low, clip_high, kl_coef;
    float *loss, *grad;   // grad: the marginals in, the gradient out
};

constexpr double kChartScore = (double)1.4426950408889634f * 0.69314718055994530942;

// Log ratios above this are taken as this (e^80 = 5.5e34 is finite in float32).
constexpr double kMaxLogRatio = 80.0;

// Sums and differences of scores are float64: log p is a difference of two
// sums of hundreds of scores, and which side of a clip border a ratio falls
// on hangs on it.
//
// The charts hold scores in log2 units, s log2(e) rounded to float32 for the
// factor, which makes every score that a tree is free to have or not
// (1 - 1.3e-8) s.  Z is then that CRF's, and a tree's own scores are taken the
// same way: what the factor does to the two cancels but for the difference
// between the tree's score and the mean (log Z alone is 1.0e-5 off for it at
// 300 words of deviation 2, 1.4e-6 without).
//
// With a gradient: a cell of the stripe has a mask of the trees that hold it (W words
// of 32 trees), set by atomic ORs in LDS, whose order cannot change the
// result and which count a repeated span once; the cell's coefficients are
// then summed in the order of the trees.  A span of every tree takes the sum
// of all coefficients, so that the gradient of a span that every tree must
// have (p = 1) is exactly zero.
struct TreeArgs {
    const int32_t *recs;   // KernelPlan::tree_recs
    int N1, G, W;
    const float *scores;
    const int32_t *trees, *counts;
    const double *z64;
    float *logp, *logZ;
    PolicyArgs p;
};

// A workgroup a record.  (A wavefront for each sentence of up to 32 words, four
// a workgroup, was slower for small batches: 8 trees of 200 sentences 19.7 us
// against 11.4, 4 of 5,000 26.1 against 27.9: the steps that one wavefront takes
// alone add up.)
template <TreeMode MODE>
__global__ __launch_bounds__(kTreeThreads) void tree_kernel(TreeArgs ta) {
    extern __shared__ __align__(16) uint32_t mask[];
    __shared__ double sums[CRF_MAX_TREES];
    __shared__ float coef[CRF_MAX_TREES + 1];
    constexpr bool GRAD = MODE != kTreeLogp;
    constexpr int NW = kTreeThreads / 64, NT = kTreeThreads;
    const PolicyArgs &a = ta.p;
    const int N1 = ta.N1, G = ta.G, W = ta.W;
    const float *scores = ta.scores;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int4 rec = reinterpret_cast<const int4 *>(ta.recs)[blockIdx.x];
    const int b = rec.x, n = rec.y, i0 = rec.z, rows = rec.w;
    if (!GRAD && i0 != 0) return;
    const int cnt = ta.counts ? min(max(ta.counts[b], 0), G) : G;
    const int R = 2 * (N1 - 1) - 1, own = 2 * n - 1;
    const size_t sent = (size_t)b * N1 * N1;
    // (as bits, which is_nan takes)
    const uint64_t zb = MODE == kTreeBack ? 0 : reinterpret_cast<const uint64_t *>(ta.z64)[b];
    const double z = __builtin_bit_cast(double, zb);
    const size_t at = (size_t)b * G + min(lane, G - 1);
    auto bits = [at](const float *x) { return reinterpret_cast<const uint32_t *>(x)[at]; };
    uint32_t advb = 0, oldb = 0, refb = 0;
    float up = 1.f;
    if constexpr (MODE == kTreePolicy) {
        advb = bits(a.adv);
        oldb = bits(a.old_logp);
        if (a.ref_logp != nullptr) refb = bits(a.ref_logp);
        if (a.grad_loss != nullptr) up = a.grad_loss[b];
    } else if constexpr (MODE == kTreeBack) {
        advb = bits(a.grad_logp);
    }
    const float adv = __builtin_bit_cast(float, advb), old = __builtin_bit_cast(float, oldb),
                ref = __builtin_bit_cast(float, refb);
    const float inv = 1.0f / (float)n;
    struct Cell {
        int i, j;
        bool ok;
    };
    auto cell_of = [&](int t) {
        int r = (int)(((float)t + 0.5f) * inv);   // t / n: t < 2^12, off by one at most
        r -= r * n > t;
        r += (r + 1) * n <= t;
        const int i = i0 + r, j = t - r * n + 1;
        return Cell{i, j, t < rows * n && j > i};
    };
    float p[kAhead];
    auto load_cells = [&](int t0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const Cell c = cell_of(t0 + u * NT);
            p[u] = c.ok ? a.grad[sent + (size_t)c.i * N1 + c.j] : 0.f;
        }
    };
    if constexpr (GRAD) {
        load_cells(tid);
        for (int t = tid; t < rows * n * W; t += NT) mask[t] = 0u;
        __syncthreads();
    }

    // A wavefront a tree, its spans' scores 64 rows at a time, kAhead such
    // pieces (of one tree or several) in flight.
    const int pieces = (own + 63) >> 6, mine = (cnt - wave + NW - 1) / NW;
    int g = wave, c = 0;   // the tree and piece that are summed next
    double acc = 0.0;
    for (int at0 = 0; at0 < mine * pieces; at0 += kAhead) {
        int2 sp[kAhead];
        float v[kAhead];
        int gu = g, cu = c;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = 64 * cu + lane;
            const bool in = gu < cnt && r < own;
            sp[u] = reinterpret_cast<const int2 *>(ta.trees)[((size_t)b * G + (in ? gu : 0)) * R + (in ? r : 0)];
            if (!(in && 0 <= sp[u].x && sp[u].x < sp[u].y && sp[u].y <= n)) sp[u].x = -1;
            if (++cu == pieces) cu = 0, gu += NW;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) v[u] = sp[u].x >= 0 ? scores[sent + (size_t)sp[u].x * N1 + sp[u].y] : 0.f;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (g >= cnt) break;
            const bool forced = sp[u].y == sp[u].x + 1 || (sp[u].x == 0 && sp[u].y == n);
            acc += (double)v[u] * (forced ? 1.0 : kChartScore);
            if constexpr (GRAD)
                if (sp[u].x >= i0 && sp[u].x < i0 + rows)
                    atomicOr(&mask[((sp[u].x - i0) * n + sp[u].y - 1) * W + (g >> 5)], 1u << (g & 31));
            if (++c == pieces) {
                acc = wave_sum(acc);
                if (lane == 0) sums[g] = acc;
                acc = 0.0;
                c = 0;
                g += NW;
            }
        }
    }
    __syncthreads();

    // The trees' terms, a lane each (G <= 64).
    if (wave == 0) {
        const bool here = lane < cnt;
        const double lp = here ? sums[lane] - z : 0.0;
        if (i0 == 0)
            if (here && ta.logp != nullptr) ta.logp[at] = or_nan(is_nan(zb), (float)lp);
        if constexpr (MODE == kTreeLogp) {
            if (lane == 0 && ta.logZ != nullptr) ta.logZ[b] = or_nan(is_nan(zb), (float)z);
        } else if constexpr (MODE == kTreeBack) {
            const float c = here ? adv : 0.f;
            const double all = wave_sum((double)c);
            if (here) coef[lane] = c;
            if (lane == 0) coef[CRF_MAX_TREES] = (float)all;
        } else {
            double term = 0.0, c = 0.0;
            if (here) {
                const double A = adv, r = exp(fmin(lp - (double)old, kMaxLogRatio));
                const double kept = fmin(fmax(r, 1.0 - (double)a.clip_low), 1.0 + (double)a.clip_high);
                const bool free = r * A <= kept * A;
                term = -(free ? r : kept) * A;
                c = free ? -r * A : 0.0;
                if (a.ref_logp != nullptr) {
                    const double q = fmin((double)ref - lp, kMaxLogRatio), e = expm1(q);
                    term += (double)a.kl_coef * (e - q);
                    c -= (double)a.kl_coef * e;
                }
            }
            // (log Z is NaN where a team's wait ran out)
            const bool lost = __any(here && (is_nan(zb) || is_nan(advb) || is_nan(oldb) || is_nan(refb)));
            const double share = cnt > 0 ? 1.0 / (double)cnt : 0.0;
            const double total = wave_sum(term) * share, all = wave_sum((double)(float)(c * share));
            if (here) coef[lane] = (float)(c * share);
            if (lane == 0) {
                coef[CRF_MAX_TREES] = or_nan(lost, (float)all);
                if (i0 == 0) a.loss[b] = or_nan(lost, (float)total);
            }
        }
    }
    if constexpr (!GRAD) return;
    __syncthreads();

    // The cells of the stripe.
    const float all = coef[CRF_MAX_TREES];
    const uint32_t full[2] = {cnt >= 32 ? ~0u : (1u << cnt) - 1u, cnt >= 64 ? ~0u : cnt > 32 ? (1u << (cnt - 32)) - 1u : 0u};
    for (int t0 = tid; t0 < rows * n; t0 += kAhead * NT) {
        if (t0 != tid) load_cells(t0);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int t = t0 + u * NT;
            const Cell c = cell_of(t);
            if (!c.ok) continue;
            float sum = 0.f;
            bool every = cnt > 0;
            for (int w = 0; w < W; ++w) {
                uint32_t m = mask[t * W + w];
                every = every && m == full[w];
                for (; m != 0; m &= m - 1) sum += coef[32 * w + __builtin_ctz(m)];
            }
            a.grad[sent + (size_t)c.i * N1 + c.j] = up * ((every ? all : sum) - all * p[u]);
        }
    }
}

// log Z of n sentences as not there, NaN.
__global__ void mark_missing(const int32_t *ids, int n, double *z64) {
    for (int t = threadIdx.x; t < n; t += blockDim.x) reinterpret_cast<uint64_t *>(z64)[ids[t]] = 0x7FF8000000000000ull;
}

}  // namespace

// The sweep.  A launch by teams that the device never holds at once writes
// nothing, and log Z would be what the workspace held before: it is NaN until
// a team has it, and with it what the pass over the trees makes of it.
static hipError_t sweep(const KernelPlan &p, const float *scores, double *z64, float *marg, hipStream_t stream) {
    if (z64 != nullptr && inside_by_teams(p)) {
        hipLaunchKernelGGL(mark_missing, dim3(1), dim3(64), 0, stream, p.inside.order_spill, (int)p.inside.n_spill, z64);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    KernelPlan q = p;
    q.z64 = z64;
    return launch_inside(q, scores, nullptr, nullptr, marg, stream);
}

// The sweep, then the pass over the trees.
template <TreeMode MODE>
static hipError_t launch_trees(const KernelPlan &p, const float *scores, const int32_t *trees, int G,
                               const int32_t *counts, double *z64, float *logp, float *logZ, const PolicyArgs &a,
                               hipStream_t stream) {
    const hipError_t e = sweep(p, scores, z64, a.grad, stream);
    if (e != hipSuccess) return e;
    const int W = (G + 31) / 32;
    const TreeArgs ta{p.tree_recs, p.n1, G, W, scores, trees, counts, z64, logp, logZ, a};
    hipLaunchKernelGGL(tree_kernel<MODE>, dim3(p.n_tree_recs), dim3(kTreeThreads),
                       MODE == kTreeLogp ? 0 : (size_t)p.tree_cells * W * 4, stream, ta);
    return hipGetLastError();
}

hipError_t launch_tree_logprobs(const KernelPlan &p, const float *scores, const int32_t *trees, int G,
                                const int32_t *counts, double *z64, float *logp, float *logZ, hipStream_t stream) {
    return launch_trees<kTreeLogp>(p, scores, trees, G, counts, z64, logp, logZ, PolicyArgs{}, stream);
}

hipError_t launch_tree_logprobs_bwd(const KernelPlan &p, const float *scores, const int32_t *trees, int G,
                                    const int32_t *counts, const float *grad_logp, float *grad, hipStream_t stream) {
    PolicyArgs a{};
    a.grad_logp = grad_logp;
    a.grad = grad;
    return launch_trees<kTreeBack>(p, scores, trees, G, counts, nullptr, nullptr, nullptr, a, stream);
}

hipError_t launch_policy_loss(const KernelPlan &p, const float *scores, const int32_t *trees, int G,
                              const int32_t *counts, const float *adv, const float *old_logp, const float *ref_logp,
                              float clip_low, float clip_high, float kl_coef, const float *grad_loss, double *z64,
                              float *loss, float *logp, float *grad, hipStream_t stream) {
    const PolicyArgs a{nullptr, adv, old_logp, ref_logp, grad_loss, clip_low, clip_high, kl_coef, loss, grad};
    return launch_trees<kTreePolicy>(p, scores, trees, G, counts, z64, logp, nullptr, a, stream);
}

}  // namespace crf
