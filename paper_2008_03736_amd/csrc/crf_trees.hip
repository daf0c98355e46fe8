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
// sentence, or per stripe of a long sentence's rows.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "crf_internal.h"

namespace crf {
namespace {

constexpr int kTreeThreads = 256;
constexpr int kTreeWords = 8192;   // mask words a workgroup holds (32 KB: five workgroups a CU)
constexpr int kAhead = 4;          // rows a lane has in flight

// Rows of a sentence of n words in a stripe whose masks of W words a cell fit
// in kTreeWords (a row holds n cells: columns 1..n), and its stripes.
__host__ __device__ inline int stripe_rows(int n, int W) { return n * W <= kTreeWords ? kTreeWords / (n * W) : 1; }
__host__ __device__ inline int stripes(int n, int W) {
    const int r = stripe_rows(n, W);
    return (n + r - 1) / r;
}
static_assert(CRF_MAX_LEN * 2 <= kTreeWords, "a row of the longest sentence fits, 64 trees");

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) v += __shfl_xor(v, k, 64);
    return v;
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
template <TreeMode MODE>
__global__ __launch_bounds__(kTreeThreads) void tree_kernel(const int32_t *__restrict__ len, int N1, int G, int W,
                                                            const float *__restrict__ scores,
                                                            const int32_t *__restrict__ trees,
                                                            const int32_t *__restrict__ counts,
                                                            const double *__restrict__ z64, float *__restrict__ logp,
                                                            float *__restrict__ logZ, PolicyArgs a) {
    extern __shared__ __align__(16) uint32_t mask[];
    __shared__ double sums[CRF_MAX_TREES];
    __shared__ float coef[CRF_MAX_TREES + 1];
    constexpr bool GRAD = MODE != kTreeLogp;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = blockIdx.x, n = len[b];
    int i0 = 0, rows = n;
    if constexpr (GRAD) {
        const int per = stripe_rows(n, W);
        i0 = (int)blockIdx.y * per;
        if (i0 >= n) return;
        rows = min(per, n - i0);
        for (int t = tid; t < rows * n * W; t += kTreeThreads) mask[t] = 0u;
        __syncthreads();
    }
    const int cnt = counts ? min(max(counts[b], 0), G) : G;
    const int R = 2 * (N1 - 1) - 1, own = 2 * n - 1;
    const size_t sent = (size_t)b * N1 * N1;
    const double z = MODE == kTreeBack ? 0.0 : z64[b];

    // A wavefront a tree: its spans' scores, a row a lane.
    for (int g = wave; g < cnt; g += kTreeThreads / 64) {
        const int2 *t = reinterpret_cast<const int2 *>(trees) + ((size_t)b * G + g) * R;
        double acc = 0.0;
        for (int r0 = lane; r0 < own; r0 += 64 * kAhead) {
            int2 sp[kAhead];
            float v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                sp[u] = t[min(r0 + 64 * u, own - 1)];
                if (r0 + 64 * u >= own || !(0 <= sp[u].x && sp[u].x < sp[u].y && sp[u].y <= n)) sp[u].x = -1;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) v[u] = sp[u].x >= 0 ? scores[sent + (size_t)sp[u].x * N1 + sp[u].y] : 0.f;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const bool forced = sp[u].y == sp[u].x + 1 || (sp[u].x == 0 && sp[u].y == n);
                acc += (double)v[u] * (forced ? 1.0 : kChartScore);
                if constexpr (GRAD)
                    if (sp[u].x >= i0 && sp[u].x < i0 + rows)
                        atomicOr(&mask[((sp[u].x - i0) * n + sp[u].y - 1) * W + (g >> 5)], 1u << (g & 31));
            }
        }
        acc = wave_sum(acc);
        if (lane == 0) sums[g] = acc;
    }
    __syncthreads();

    // The trees' terms, a lane each (G <= 64).
    if (wave == 0) {
        const bool here = lane < cnt;
        const size_t at = (size_t)b * G + lane;
        const double lp = here ? sums[lane] - z : 0.0;
        if (!GRAD || blockIdx.y == 0)
            if (here && logp != nullptr) logp[at] = (float)lp;
        if constexpr (MODE == kTreeLogp) {
            if (lane == 0 && logZ != nullptr) logZ[b] = (float)z;
        } else if constexpr (MODE == kTreeBack) {
            const float c = here ? a.grad_logp[at] : 0.f;
            const double all = wave_sum((double)c);
            if (here) coef[lane] = c;
            if (lane == 0) coef[CRF_MAX_TREES] = (float)all;
        } else {
            double term = 0.0, c = 0.0;
            if (here) {
                const double A = a.adv[at], r = exp(fmin(lp - (double)a.old_logp[at], kMaxLogRatio));
                const double kept = fmin(fmax(r, 1.0 - (double)a.clip_low), 1.0 + (double)a.clip_high);
                const bool free = r * A <= kept * A;
                term = -(free ? r : kept) * A;
                c = free ? -r * A : 0.0;
                if (a.ref_logp != nullptr) {
                    const double q = fmin((double)a.ref_logp[at] - lp, kMaxLogRatio), e = expm1(q);
                    term += (double)a.kl_coef * (e - q);
                    c -= (double)a.kl_coef * e;
                }
            }
            const double share = cnt > 0 ? 1.0 / (double)cnt : 0.0;
            const double total = wave_sum(term) * share, all = wave_sum((double)(float)(c * share));
            if (here) coef[lane] = (float)(c * share);
            if (lane == 0) {
                coef[CRF_MAX_TREES] = (float)all;
                if (blockIdx.y == 0) a.loss[b] = (float)total;
            }
        }
    }
    if constexpr (!GRAD) return;
    __syncthreads();

    // The cells of the stripe.
    const float all = coef[CRF_MAX_TREES], gl = a.grad_loss ? a.grad_loss[b] : 1.0f;
    const float inv = 1.0f / (float)n;
    const uint32_t full[2] = {cnt >= 32 ? ~0u : (1u << cnt) - 1u, cnt >= 64 ? ~0u : cnt > 32 ? (1u << (cnt - 32)) - 1u : 0u};
    for (int t = tid; t < rows * n; t += kTreeThreads) {
        int r = (int)(((float)t + 0.5f) * inv);   // t / n: t < 2^13, off by one at most
        r -= r * n > t;
        r += (r + 1) * n <= t;
        const int i = i0 + r, j = t - r * n + 1;
        if (j <= i) continue;
        float sum = 0.f;
        bool every = cnt > 0;
        for (int w = 0; w < W; ++w) {
            uint32_t m = mask[t * W + w];
            every = every && m == full[w];
            for (; m != 0; m &= m - 1) sum += coef[32 * w + __builtin_ctz(m)];
        }
        float *cell = a.grad + sent + (size_t)i * N1 + j;
        *cell = gl * ((every ? all : sum) - all * *cell);
    }
}

}  // namespace

static hipError_t sweep(const KernelPlan &p, const float *scores, double *z64, float *marg, hipStream_t stream) {
    KernelPlan q = p;
    q.z64 = z64;
    return launch_inside(q, scores, nullptr, nullptr, marg, stream);
}

hipError_t launch_tree_logprobs(const KernelPlan &p, const float *scores, const int32_t *trees, int G,
                                const int32_t *counts, double *z64, float *logp, float *logZ, hipStream_t stream) {
    const hipError_t e = sweep(p, scores, z64, nullptr, stream);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(tree_kernel<kTreeLogp>, dim3(p.B), dim3(kTreeThreads), 0, stream, p.len, p.n1, G, 1, scores, trees,
                       counts, z64, logp, logZ, PolicyArgs{});
    return hipGetLastError();
}

static hipError_t launch_gradient(void (*kernel)(const int32_t *, int, int, int, const float *, const int32_t *,
                                                 const int32_t *, const double *, float *, float *, PolicyArgs),
                                  const KernelPlan &p, int max_len, const float *scores, const int32_t *trees, int G,
                                  const int32_t *counts, double *z64, float *logp, const PolicyArgs &a,
                                  hipStream_t stream) {
    const hipError_t e = sweep(p, scores, z64, a.grad, stream);
    if (e != hipSuccess) return e;
    const int W = (G + 31) / 32;
    int most = 1, words = 0;
    for (int n = 1; n <= max_len; ++n) {
        most = std::max(most, stripes(n, W));
        words = std::max(words, std::min(n, stripe_rows(n, W)) * n * W);
    }
    hipLaunchKernelGGL(kernel, dim3(p.B, most), dim3(kTreeThreads), (size_t)words * 4, stream, p.len, p.n1, G, W, scores,
                       trees, counts, z64, logp, nullptr, a);
    return hipGetLastError();
}

hipError_t launch_tree_logprobs_bwd(const KernelPlan &p, int max_len, const float *scores, const int32_t *trees, int G,
                                    const int32_t *counts, const float *grad_logp, float *grad, hipStream_t stream) {
    PolicyArgs a{};
    a.grad_logp = grad_logp;
    a.grad = grad;
    return launch_gradient(tree_kernel<kTreeBack>, p, max_len, scores, trees, G, counts, nullptr, nullptr, a, stream);
}

hipError_t launch_policy_loss(const KernelPlan &p, int max_len, const float *scores, const int32_t *trees, int G,
                              const int32_t *counts, const float *adv, const float *old_logp, const float *ref_logp,
                              float clip_low, float clip_high, float kl_coef, const float *grad_loss, double *z64,
                              float *loss, float *logp, float *grad, hipStream_t stream) {
    const PolicyArgs a{nullptr, adv, old_logp, ref_logp, grad_loss, clip_low, clip_high, kl_coef, loss, grad};
    return launch_gradient(tree_kernel<kTreePolicy>, p, max_len, scores, trees, G, counts, z64, logp, a, stream);
}

}  // namespace crf
