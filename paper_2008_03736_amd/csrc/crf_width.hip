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
//
// 5,000 sentences, one label: 9.6 us forward; 15.4 back, and 4 to join the shares.
// Their rows are 12 cells long on the average, at odd places: 25 MB of lines are
// read for 7.9 MB of cells, both ways; back, a thread's 32 loads a block are all
// issued, whatever the rows' lengths.  100 sentences of 138 labels: 12.3 us forward (3.7 TB/s
// of the cells); 12.3 back and 4.2, as long as the few passes of a workgroup.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "crf_internal.h"

namespace crf {
namespace {

constexpr int kWidthThreads = 256;
constexpr int kFewBuckets = 64;
constexpr int kMaxWidth = 1023;      // a sentence's most words
// Workgroups that a call aims at.  Forward, 100 sentences of 138 labels: 19.6 us at
// 1,024, 14.8 at 2,048, 12.7 at 4,096.  Back, where each adds a share to what is
// joined: 18.4 us both at 1,024, 16.4 at 2,048, 19.0 at 4,096.
constexpr int kWidthGroups = 4096, kWidthSumGroups = 2048;
constexpr int kWidthShares = 1024;   // most shares (5,000 sentences: 18.9 us at 512, 15.4, 16.6 at 2,048)

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
    typename Cells<V>::type v;
    const int k = bucket[w];
    const bool there = k >= 0 && k < K;
    const float *row = table + (size_t)(there ? k : 0) * L + label;
    if constexpr (V == 1) {
        v = there ? row[0] : 0.f;
    } else {
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] = there ? row[q] : 0.f;
    }
    return v;
}

// The rows of a block of posts that are group r's, a row's threads: with P = 64 a
// wavefront's run of them, so that what is looked up by a row comes by scalar
// loads, many rows in each.  (A load a row keeps the scalar caches busy for 4 us
// more with 100 sentences of 138 labels; with P = 16 runs are 1 us slower.)
template <int P>
__device__ __forceinline__ int row_group() {
    const int r = threadIdx.x / P;
    return P == 64 ? __builtin_amdgcn_readfirstlane(r) : r;
}
template <int P>
__device__ __forceinline__ int row_of(int group, int m) {
    constexpr int kRows = kWidthThreads / P, kMine = kBiaRows / kRows;
    return P == 64 ? group * kMine + m : group + m * kRows;
}

// A workgroup takes a block of posts and every gridDim.y-th group of N tiles of P
// places.
template <int V, int P, int N>
__global__ __launch_bounds__(kWidthThreads) void width_kernel(const int32_t *__restrict__ posts,
                                                              const int64_t *__restrict__ post_cells, int L, int K,
                                                              const float *__restrict__ table,
                                                              const int32_t *__restrict__ bucket, const float *scores,
                                                              float *out) {
    typedef typename Cells<V>::type cells;
    constexpr int kRows = kWidthThreads / P, kMine = kBiaRows / kRows;
    const int32_t *rest = posts + (size_t)blockIdx.x * kPostRec + kBiaRows;
    const int64_t *at = post_cells + (size_t)blockIdx.x * kBiaRows;
    const int group = row_group<P>(), per = L / V;   // (per: places of a width)
    int wide[kMine], most = 0;
    size_t base[kMine];
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
        wide[m] = rest[row_of<P>(group, m)];
        base[m] = (size_t)at[row_of<P>(group, m)] * L;
        most = max(most, wide[m]);
    }
    for (int e0 = blockIdx.y * N * P + threadIdx.x % P; e0 < most * per; e0 += gridDim.y * N * P) {
        int w[N];
        size_t off[N];
        cells v[N][kMine], bias[N];
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int e = e0 + t * P;
            w[t] = e / per;
            off[t] = (size_t)(w[t] + 1) * L + (e - w[t] * per) * V;
#pragma unroll
            for (int m = 0; m < kMine; ++m)
                if (w[t] < wide[m]) v[t][m] = *reinterpret_cast<const cells *>(scores + base[m] + off[t]);
        }
#pragma unroll
        for (int t = 0; t < N; ++t)   // (on its way beside the scores; widths past the row's are not there)
            bias[t] = entry<V>(table, bucket, K, L, min(w[t] + 1, most), (e0 + t * P - w[t] * per) * V);
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int m = 0; m < kMine; ++m)
                if (w[t] < wide[m]) *reinterpret_cast<cells *>(out + base[m] + off[t]) = v[t][m] + bias[t];
    }
}

// A workgroup takes N tiles of P places, from tile N blockIdx.y on, and every
// gridDim.x-th block of posts.
template <int V, int P, int N>
__global__ __launch_bounds__(kWidthThreads) void width_bwd_kernel(const int32_t *__restrict__ posts,
                                                                  const int64_t *__restrict__ post_cells, int n_posts,
                                                                  int widest, int L, const float *__restrict__ grad,
                                                                  const int32_t *__restrict__ bucket, int K,
                                                                  float *__restrict__ grad_scores,
                                                                  float *__restrict__ parts) {
    typedef typename Cells<V>::type cells;
    constexpr int kRows = kWidthThreads / P, kMine = kBiaRows / kRows;
    __shared__ cells sums[kRows][N * P];
    __shared__ int buckets[P == 16 ? N * P + 1 : 1];
    const int group = row_group<P>(), c = threadIdx.x % P, per = L / V, e0 = blockIdx.y * N * P + c;
    int w[N];
    size_t off[N];
    cells sum[N];
#pragma unroll
    for (int t = 0; t < N; ++t) {
        const int e = e0 + t * P;
        w[t] = e / per;
        off[t] = (size_t)(w[t] + 1) * L + (e - w[t] * per) * V;
        sum[t] = 0.f;
    }
    // (the next block's rows are looked up while this one's cells are read)
    int wide[kMine], wide1[kMine];
    size_t base[kMine], base1[kMine];
    auto look = [&](int block) {
        const int32_t *rest = posts + (size_t)block * kPostRec + kBiaRows;
        const int64_t *at = post_cells + (size_t)block * kBiaRows;
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            wide1[m] = rest[row_of<P>(group, m)];
            base1[m] = (size_t)at[row_of<P>(group, m)] * L;
        }
    };
    look(blockIdx.x);
    for (int block = blockIdx.x; block < n_posts; block += gridDim.x) {
#pragma unroll
        for (int m = 0; m < kMine; ++m) wide[m] = wide1[m], base[m] = base1[m];
        if (block + (int)gridDim.x < n_posts) look(block + (int)gridDim.x);
        cells v[N][kMine];
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int m = 0; m < kMine; ++m) {
                v[t][m] = 0.f;
                if (w[t] < wide[m]) v[t][m] = *reinterpret_cast<const cells *>(grad + base[m] + off[t]);
            }
        if (grad_scores != nullptr) {
#pragma unroll
            for (int t = 0; t < N; ++t)
#pragma unroll
                for (int m = 0; m < kMine; ++m)
                    if (w[t] < wide[m]) *reinterpret_cast<cells *>(grad_scores + base[m] + off[t]) = v[t][m];
        }
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int m = 0; m < kMine; ++m) sum[t] += v[t][m];
    }
    if (parts == nullptr) return;
#pragma unroll
    for (int t = 0; t < N; ++t) sums[group][t * P + c] = sum[t];
    __syncthreads();
    // to parts[share][width's label], or parts[bucket's label][share] (K > 0)
    const int shares = gridDim.x * (K > 0 ? gridDim.y : 1), share = K > 0 ? blockIdx.y * gridDim.x + blockIdx.x : blockIdx.x;
    const int first = blockIdx.y * N * P;
    for (int q = threadIdx.x; q < N * P; q += kWidthThreads) {
        cells s = sums[0][q];
        for (int r = 1; r < kRows; ++r) s += sums[r][q];
        if (P == 16 && K > 0) {
            sums[0][q] = s;
        } else if (first + q < widest * per) {
            *reinterpret_cast<cells *>(parts + (size_t)share * widest * L + (size_t)(first + q) * V) = s;
        }
    }
    if constexpr (P == 16) {
        if (K == 0) return;
        // the widths that this workgroup has places of, and their buckets
        const int w0 = first / per, w1 = min((first + N * P - 1) / per, widest - 1);
        for (int q = threadIdx.x; w0 + q <= w1; q += kWidthThreads) buckets[q] = bucket[w0 + q + 1];
        __syncthreads();
        // sixteen lanes a bucket's label, every sixteenth width each
        for (int q = threadIdx.x / 16; q < K * L; q += kWidthThreads / 16) {
            const int k = q / L, label = q - k * L, part = label / V, h = label - part * V;
            float s = 0.f;
            for (int v = w0 + threadIdx.x % 16; v <= w1; v += 16) {
                const int place = v * per + part - first;
                if (buckets[v - w0] == k && place >= 0 && place < N * P)
                    s += reinterpret_cast<const float *>(sums[0])[place * V + h];
            }
#pragma unroll
            for (int x = 1; x < 16; x *= 2) s += __shfl_xor(s, x, 16);
            if (threadIdx.x % 16 == 0) parts[(size_t)q * shares + share] = s;
        }
    }
}

// A bucket's widths and the shares of the rows added up in a fixed order: J
// labels a workgroup, thread (l, p) every kLanes-th of the bucket's (width,
// share) pairs.
constexpr int kJoinThreads = 1024;
template <int J>
__global__ __launch_bounds__(kJoinThreads) void width_join_kernel(const float *__restrict__ parts, int shares, int widest,
                                                                  int L, const int32_t *__restrict__ bucket,
                                                                  bool by_bucket, float *__restrict__ grad_table) {
    constexpr int kLanes = kJoinThreads / J;
    __shared__ float part[kLanes][J + 1];
    __shared__ uint16_t widths[1024];   // the bucket's, in order
    __shared__ int before[kJoinThreads / 64];
    static_assert(kMaxWidth <= 1024 && kMaxWidth <= kJoinThreads, "a thread a width");
    const int k = blockIdx.x, tid = threadIdx.x, l = tid % J, p = tid / J, label = blockIdx.y * J + l;
    // the rows of parts that are the bucket's: its widths, or itself
    const bool mine = by_bucket ? tid == k : tid < widest && bucket[tid + 1] == k;
    const uint64_t all = __ballot(mine);
    if ((tid & 63) == 0) before[tid >> 6] = __popcll(all);
    __syncthreads();
    int count = 0, at = 0;
    for (int w = 0; w < kJoinThreads / 64; ++w) {
        if (w == tid >> 6) at = count;
        count += before[w];
    }
    if (mine) widths[at + __popcll(all & ((1ull << (tid & 63)) - 1))] = (uint16_t)tid;
    __syncthreads();
    float s = 0.f;
    if (label < L) {
#pragma unroll 8
        for (int q = p; q < count * shares; q += kLanes) {
            const int w = q / shares, share = q - w * shares;
            s += by_bucket ? parts[((size_t)widths[w] * L + label) * shares + share]
                           : parts[((size_t)share * widest + widths[w]) * L + label];
        }
    }
    part[p][l] = s;
    __syncthreads();
    for (int half = kLanes / 2; half > 0; half /= 2) {
        if (p < half) part[p][l] += part[p + half][l];
        __syncthreads();
    }
    if (p == 0 && label < L) grad_table[(size_t)k * L + label] = part[0][l];
}

// Places of a tile, and tiles a workgroup has in flight: rows of one label are
// short, those of many long.
bool many_labels(int L) { return L >= 16; }
constexpr int tiles_in_flight(int V, int P) { return P == 64 ? 1 : 8 / V; }
int tiles(int widest, int L, int V) {
    const int P = many_labels(L) ? 64 : 16;
    return (int)(((int64_t)widest * (L / V) + P - 1) / P);
}
// Labels a thread takes: what the arrays' alignment allows.
int labels_each(int L, const void *a, const void *b) {
    const uintptr_t at = (uintptr_t)a | (uintptr_t)b;
    return L % 4 == 0 && at % 16 == 0 ? 4 : L % 2 == 0 && at % 8 == 0 ? 2 : 1;
}
// Shares of the rows; with few labels and buckets the workgroups add up a
// bucket's widths themselves.
int tile_groups(int widest, int L, int V) {
    const int N = many_labels(L) ? 1 : 8 / V;
    return (tiles(widest, L, V) + N - 1) / N;
}
int width_shares(const KernelPlan &p, int widest, int L) {
    const int t = tile_groups(widest, L, 1);
    return std::min({p.n_posts, kWidthShares, std::max(8, (kWidthSumGroups + t - 1) / t)});
}
bool by_bucket(int L, int K) { return !many_labels(L) && K <= kFewBuckets; }

template <int V, int P>
void launch_width_v(const KernelPlan &p, int widest, int L, const float *table, const int32_t *bucket, int K,
                    const float *scores, float *out, hipStream_t stream) {
    constexpr int N = P == 64 ? 1 : 4 / V;
    const int y = std::max(1, std::min((tiles(widest, L, V) + N - 1) / N, kWidthGroups / p.n_posts));
    hipLaunchKernelGGL((width_kernel<V, P, N>), dim3(p.n_posts, y), dim3(kWidthThreads), 0, stream, p.posts, p.post_cells, L,
                       K, table, bucket, scores, out);
}
template <int V, int P>
void launch_width_bwd_v(const KernelPlan &p, int widest, int L, const float *grad, float *grad_scores, float *parts,
                        const int32_t *bucket, int K, hipStream_t stream) {
    constexpr int N = tiles_in_flight(V, P);
    hipLaunchKernelGGL((width_bwd_kernel<V, P, N>), dim3(width_shares(p, widest, L), tile_groups(widest, L, V)),
                       dim3(kWidthThreads), 0, stream, p.posts, p.post_cells, p.n_posts, widest, L, grad, bucket,
                       by_bucket(L, K) ? K : 0, grad_scores, parts);
}

template <int J>
void launch_join(const KernelPlan &p, int widest, int L, int V, const int32_t *bucket, int K, const float *parts,
                 float *grad_table, hipStream_t stream) {
    const bool own = by_bucket(L, K);
    hipLaunchKernelGGL(width_join_kernel<J>, dim3(K, (L + J - 1) / J), dim3(kJoinThreads), 0, stream, parts,
                       width_shares(p, widest, L) * (own ? tile_groups(widest, L, V) : 1), widest, L, bucket, own, grad_table);
}

}  // namespace

int64_t width_bwd_bytes(const KernelPlan &p, int widest, int L) {
    // (by width, or by bucket: at most kFewBuckets for each group of tiles of one label)
    const int64_t rows = many_labels(L) ? widest : std::max(widest, kFewBuckets * tile_groups(widest, L, 1));
    return ((int64_t)width_shares(p, widest, L) * rows * L * 4 + 255) / 256 * 256;
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
            p, widest, L, grad, grad_scores, parts, bucket, K, stream);
    else
        (V == 4 ? launch_width_bwd_v<4, 16> : V == 2 ? launch_width_bwd_v<2, 16> : launch_width_bwd_v<1, 16>)(
            p, widest, L, grad, grad_scores, parts, bucket, K, stream);
    if (grad_table != nullptr)
        (L == 1 ? launch_join<1> : L < 16 ? launch_join<4> : launch_join<16>)(p, widest, L, V, bucket, K, parts, grad_table, stream);
    return hipGetLastError();
}

}  // namespace crf
