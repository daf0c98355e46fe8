// crf_width.hip -- a learned bias by a span's width, and its table's gradient.
//
//     out(i,j,l) = s(i,j,l) + T[bucket[j - i]][l],
//     dT[k][l] = sum of dL/dout(i,j,l) over the spans with bucket[j - i] = k.
//
// Memory-bound: 8 bytes a cell forward, 4 back (8 with the scores' own
// gradient).  A row's cells (i, i+1), (i, i+2) ... and their labels are
// neighbours in memory, and place e of a row, e = (width - 1) L + label, means
// the same table entry in every row of every sentence.  So a thread keeps to
// its place (V labels of one width) and goes down the rows: its bias is a
// register, and the gradient's sum over rows one too.  The plan's lists of fence
// posts give the rows.  Sums run in a fixed order, in 32 bits: rows of a thread,
// threads of a place in LDS, then workgroups and widths of a bucket.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "crf_internal.h"

namespace crf {
namespace {

constexpr int kWidthThreads = 256;
constexpr int kWidthGroups = 2048;   // workgroups that fill the chip
constexpr int kWidthShares = 512;    // most shares of the rows whose sums are joined

template <int V>
struct Cells;
template <>
struct Cells<1> {
    typedef float type;
};
template <>
struct Cells<2> {
    typedef float type __attribute__((ext_vector_type(2)));
};
template <>
struct Cells<4> {
    typedef float type __attribute__((ext_vector_type(4)));
};

// The table's entries of a place (0 where its width has no bucket).
template <int V>
__device__ __forceinline__ typename Cells<V>::type entry(const float *table, const int32_t *bucket, int K, int L, int w,
                                                         int label) {
    typename Cells<V>::type v = 0.f;
    const int k = bucket[w];
    if (k >= 0 && k < K) {
        const float *row = table + (size_t)k * L + label;
        if constexpr (V == 1) {
            v = row[0];
        } else {
#pragma unroll
            for (int q = 0; q < V; ++q) v[q] = row[q];
        }
    }
    return v;
}

// A workgroup takes a block of posts and every gridDim.y-th tile of P places.
template <int V, int P>
__global__ __launch_bounds__(kWidthThreads) void width_kernel(const int32_t *__restrict__ posts,
                                                              const int64_t *__restrict__ post_cells, int widest, int L,
                                                              int K, const float *__restrict__ table,
                                                              const int32_t *__restrict__ bucket,
                                                              const float *scores, float *out) {
    typedef typename Cells<V>::type cells;
    constexpr int kRows = kWidthThreads / P, kMine = kBiaRows / kRows;
    const int32_t *rest = posts + (size_t)blockIdx.x * kPostRec + kBiaRows;
    const int64_t *at = post_cells + (size_t)blockIdx.x * kBiaRows;
    const int r0 = threadIdx.x / P, per = L / V;   // places of a width
    int wide[kMine], most = 0;
    size_t base[kMine];
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
        wide[m] = rest[r0 + m * kRows];
        base[m] = (size_t)at[r0 + m * kRows] * L;
        most = max(most, wide[m]);
    }
    for (int e = blockIdx.y * P + threadIdx.x % P; e < most * per; e += gridDim.y * P) {
        const int w = e / per, label = (e - w * per) * V;
        const cells bias = entry<V>(table, bucket, K, L, w + 1, label);
        const size_t off = (size_t)(w + 1) * L + label;
        cells v[kMine];
#pragma unroll
        for (int m = 0; m < kMine; ++m)
            if (w < wide[m]) v[m] = *reinterpret_cast<const cells *>(scores + base[m] + off);
#pragma unroll
        for (int m = 0; m < kMine; ++m)
            if (w < wide[m]) *reinterpret_cast<cells *>(out + base[m] + off) = v[m] + bias;
    }
}

// A workgroup takes tile blockIdx.y of P places and every gridDim.x-th block of posts.
template <int V, int P>
__global__ __launch_bounds__(kWidthThreads) void width_bwd_kernel(const int32_t *__restrict__ posts,
                                                                  const int64_t *__restrict__ post_cells, int n_posts,
                                                                  int widest, int L, const float *__restrict__ grad,
                                                                  float *__restrict__ grad_scores,
                                                                  float *__restrict__ parts) {
    typedef typename Cells<V>::type cells;
    constexpr int kRows = kWidthThreads / P, kMine = kBiaRows / kRows;
    __shared__ cells sums[kRows][P];
    const int r0 = threadIdx.x / P, c = threadIdx.x % P, per = L / V;
    const int e = blockIdx.y * P + c, w = e / per, label = (e - w * per) * V;
    const size_t off = (size_t)(w + 1) * L + label;
    cells sum = 0.f;
    for (int block = blockIdx.x; block < n_posts; block += gridDim.x) {
        const int32_t *rest = posts + (size_t)block * kPostRec + kBiaRows;
        const int64_t *at = post_cells + (size_t)block * kBiaRows;
        cells v[kMine];
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            const int r = r0 + m * kRows;
            v[m] = 0.f;
            if (w < rest[r]) {
                const size_t cell = (size_t)at[r] * L + off;
                v[m] = *reinterpret_cast<const cells *>(grad + cell);
                if (grad_scores != nullptr) *reinterpret_cast<cells *>(grad_scores + cell) = v[m];
            }
        }
#pragma unroll
        for (int m = 0; m < kMine; ++m) sum += v[m];
    }
    if (parts == nullptr) return;
    sums[r0][c] = sum;
    __syncthreads();
    for (int half = kRows / 2; half > 0; half /= 2) {
        if (r0 < half) sums[r0][c] += sums[r0 + half][c];
        __syncthreads();
    }
    if (r0 == 0 && e < widest * per)
        *reinterpret_cast<cells *>(parts + ((size_t)blockIdx.x * widest * per + e) * V) = sums[0][c];
}

// A bucket's widths and the shares of the rows added up: 16 labels a workgroup,
// thread (l, p) every 16th of the bucket's (width, share) pairs.
constexpr int kJoinLabels = 16, kJoinLanes = 16;
__global__ __launch_bounds__(kJoinLabels *kJoinLanes) void width_join_kernel(const float *__restrict__ parts, int shares,
                                                                             int widest, int L,
                                                                             const int32_t *__restrict__ bucket,
                                                                             float *__restrict__ grad_table) {
    __shared__ float part[kJoinLanes][kJoinLabels + 1];
    const int k = blockIdx.x, l = threadIdx.x % kJoinLabels, p = threadIdx.x / kJoinLabels;
    const int label = blockIdx.y * kJoinLabels + l;
    float s = 0.f;
    if (label < L)
        for (int w = 0; w < widest; ++w) {
            if (bucket[w + 1] != k) continue;
#pragma unroll 4
            for (int q = p; q < shares; q += kJoinLanes) s += parts[((size_t)q * widest + w) * L + label];
        }
    part[p][l] = s;
    __syncthreads();
    for (int half = kJoinLanes / 2; half > 0; half /= 2) {
        if (p < half) part[p][l] += part[p + half][l];
        __syncthreads();
    }
    if (p == 0 && label < L) grad_table[(size_t)k * L + label] = part[0][l];
}

// Places of a tile: rows of one label are short, those of many long.
bool many_labels(int L) { return L >= 16; }
int tiles(int widest, int L, int V) { return (int)(((int64_t)widest * (L / V) + (many_labels(L) ? 63 : 15)) / (many_labels(L) ? 64 : 16)); }
// Labels a thread takes: what the arrays' alignment allows.
int labels_each(int L, const void *a, const void *b) {
    const uintptr_t at = (uintptr_t)a | (uintptr_t)b;
    return L % 4 == 0 && at % 16 == 0 ? 4 : L % 2 == 0 && at % 8 == 0 ? 2 : 1;
}
int width_shares(const KernelPlan &p, int widest, int L) {
    const int t = tiles(widest, L, 1);
    return std::min({p.n_posts, kWidthShares, std::max(8, (2 * kWidthGroups + t - 1) / t)});
}

template <int V, int P>
void launch_width_v(const KernelPlan &p, int widest, int L, const float *table, const int32_t *bucket, int K,
                    const float *scores, float *out, hipStream_t stream) {
    const int y = std::max(1, std::min(tiles(widest, L, V), kWidthGroups / p.n_posts));
    hipLaunchKernelGGL((width_kernel<V, P>), dim3(p.n_posts, y), dim3(kWidthThreads), 0, stream, p.posts, p.post_cells,
                       widest, L, K, table, bucket, scores, out);
}
template <int V, int P>
void launch_width_bwd_v(const KernelPlan &p, int widest, int L, const float *grad, float *grad_scores, float *parts,
                        hipStream_t stream) {
    hipLaunchKernelGGL((width_bwd_kernel<V, P>), dim3(width_shares(p, widest, L), tiles(widest, L, V)), dim3(kWidthThreads),
                       0, stream, p.posts, p.post_cells, p.n_posts, widest, L, grad, grad_scores, parts);
}

}  // namespace

int64_t width_bwd_bytes(const KernelPlan &p, int widest, int L) {
    return ((int64_t)width_shares(p, widest, L) * widest * L * 4 + 255) / 256 * 256;
}

hipError_t launch_width(const KernelPlan &p, int widest, int L, const float *table, const int32_t *bucket, int K,
                        const float *scores, float *out, hipStream_t stream) {
    const int V = labels_each(L, scores, out);
    if (many_labels(L))
        (V == 4 ? launch_width_v<4, 64> : V == 2 ? launch_width_v<2, 64> : launch_width_v<1, 64>)(p, widest, L, table, bucket,
                                                                                              K, scores, out, stream);
    else
        (V == 4 ? launch_width_v<4, 16> : V == 2 ? launch_width_v<2, 16> : launch_width_v<1, 16>)(p, widest, L, table, bucket,
                                                                                              K, scores, out, stream);
    return hipGetLastError();
}

hipError_t launch_width_bwd(const KernelPlan &p, int widest, int L, const float *grad, const int32_t *bucket, int K,
                            float *grad_scores, float *grad_table, char *ws, hipStream_t stream) {
    float *parts = grad_table != nullptr ? reinterpret_cast<float *>(ws) : nullptr;
    const int V = labels_each(L, grad, grad_scores);
    if (many_labels(L))
        (V == 4 ? launch_width_bwd_v<4, 64> : V == 2 ? launch_width_bwd_v<2, 64> : launch_width_bwd_v<1, 64>)(
            p, widest, L, grad, grad_scores, parts, stream);
    else
        (V == 4 ? launch_width_bwd_v<4, 16> : V == 2 ? launch_width_bwd_v<2, 16> : launch_width_bwd_v<1, 16>)(
            p, widest, L, grad, grad_scores, parts, stream);
    if (grad_table != nullptr)
        hipLaunchKernelGGL(width_join_kernel, dim3(K, (L + kJoinLabels - 1) / kJoinLabels), dim3(kJoinLabels * kJoinLanes), 0,
                           stream, parts, width_shares(p, widest, L), widest, L, bucket, grad_table);
    return hipGetLastError();
}

}  // namespace crf
