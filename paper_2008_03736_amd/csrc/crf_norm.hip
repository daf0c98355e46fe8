// crf_norm.hip -- layer norm of fence-post rows, and its backward pass.
//
// With m and v the mean and the variance of a row's d entries, r = 1 / sqrt(v + eps)
// and h = (x - m) r,
//     y = h gamma + beta,
//     dx = r (u - mean(u) - h mean(u h)),   u = dy gamma,
//     dgamma = sum of dy h over the rows,   dbeta = sum of dy.
//
// Memory-bound: the rows are read once and written once.  A row lies in the registers
// of G lanes, eight entries each, so that its mean, its variance (of the deviations,
// not of squares) and the two means of the backward pass are sums over lanes, in 32
// bits.  A mean far past the deviations costs no digits: what its rounding leaves in
// them is their own mean, which is summed beside their squares and taken off both
// (means of 1,000 deviations: dgamma off by 1e-4 without it, by 1e-7 with it, for 0.3
// us of 62 and no more of d = 8,192).  The backward pass takes the statistics from x
// again, which it has to read anyway, and nothing is kept for it.  G is the least of
// 16 .. 1024 whose lanes hold a row: several rows to a wavefront, or several
// wavefronts to a row, which then meet in LDS.  The plan's lists of fence posts give
// the rows, so that padded ones cost nothing.
//
// 5,000 sentences of d = 500 in bf16: 54 us forward (5.0 TB/s, a large copy 5.1), 89
// back (4.6 TB/s) and 5 for joining the shares of dgamma and dbeta; 24 paragraphs of
// d = 4,096 in float32 46 and 5 back; a sentence alone 3, a launch.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "crf_internal.h"
#include "crf_rows.h"

namespace crf {
namespace {

// Most workgroups of 256 threads, forward (24 paragraphs of d = 8,192: 60 us with
// a workgroup for every four rows, 43 so) and backward, where each adds a share to
// the sums that are joined: for rows within a wavefront (5,000 sentences of d =
// 500: 98 us at 1,024 with two rows in flight, 95.6 at 1,280, 94.5), and for rows of
// several (24 paragraphs of d = 4,096 in float32: 59.4 us, 73.2 at 1,280, 67.7 at
// 1,536).
constexpr int kNormMost = 2048, kNormMostBwd = 1536, kNormMostBwdWide = 1024;

__host__ __device__ constexpr int norm_threads(int G) { return G > 256 ? G : 256; }

// Pieces of rows: bf16 rows start at multiples of 8 bytes, float32 ones of 4.
typedef uint32_t u32x4_a8 __attribute__((ext_vector_type(4), aligned(8)));
typedef uint32_t u32x2_a8 __attribute__((ext_vector_type(2), aligned(8)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }

// Entries k .. k + 7 of a row (zeros past d, a multiple of 4), as they lie in memory ...
template <typename T>
struct Raw;
template <>
struct Raw<uint16_t> {
    u32x4_a8 v = u32x4_a8{0u, 0u, 0u, 0u};
    __device__ __forceinline__ void load(const uint16_t *row, int k, int d) {
        if (k + 8 <= d) {
            v = *reinterpret_cast<const u32x4_a8 *>(row + k);
        } else if (k < d) {
            const u32x2_a8 a = *reinterpret_cast<const u32x2_a8 *>(row + k);
            v = u32x4_a8{a.x, a.y, 0u, 0u};
        }
    }
    __device__ __forceinline__ void widen(float (&f)[8]) const {
#pragma unroll
        for (int q = 0; q < 4; ++q) f[2 * q] = low(v[q]), f[2 * q + 1] = high(v[q]);
    }
};
template <>
struct Raw<float> {
    f32x4_a4 v[2] = {f32x4_a4{0.f, 0.f, 0.f, 0.f}, f32x4_a4{0.f, 0.f, 0.f, 0.f}};
    __device__ __forceinline__ void load(const float *row, int k, int d) {
        if (k < d) v[0] = *reinterpret_cast<const f32x4_a4 *>(row + k);
        if (k + 4 < d) v[1] = *reinterpret_cast<const f32x4_a4 *>(row + k + 4);
    }
    __device__ __forceinline__ void widen(float (&f)[8]) const {
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] = v[q >> 2][q & 3];
    }
};
// ... and back.
__device__ __forceinline__ void store(uint16_t *row, int k, int d, const float (&f)[8]) {
    const u32x4_a8 v = {two_bf16(f[0], f[1]), two_bf16(f[2], f[3]), two_bf16(f[4], f[5]), two_bf16(f[6], f[7])};
    if (k + 8 <= d)
        *reinterpret_cast<u32x4_a8 *>(row + k) = v;
    else if (k < d)
        *reinterpret_cast<u32x2_a8 *>(row + k) = u32x2_a8{v.x, v.y};
}
__device__ __forceinline__ void store(float *row, int k, int d, const float (&f)[8]) {
    if (k < d) *reinterpret_cast<f32x4_a4 *>(row + k) = f32x4_a4{f[0], f[1], f[2], f[3]};
    if (k + 4 < d) *reinterpret_cast<f32x4_a4 *>(row + k + 4) = f32x4_a4{f[4], f[5], f[6], f[7]};
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}
// The sum of v over the G lanes of a row, in every one of them (each adds in
// the same order).  G > 64: the row's wavefronts meet in `slots`, a place a
// wavefront; the next sum but one may use them again.
template <int G, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float *slots) {
#pragma unroll
    for (int q = 0; q < N; ++q) {
        v[q] += dpp<0xB1>(v[q]);    // quad_perm(1, 0, 3, 2)
        v[q] += dpp<0x4E>(v[q]);    // quad_perm(2, 3, 0, 1)
        v[q] += dpp<0x141>(v[q]);   // row_half_mirror
        v[q] += dpp<0x140>(v[q]);   // row_mirror
        if constexpr (G >= 32) {
            const auto h = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v[q]),
                                                            __builtin_bit_cast(uint32_t, v[q]), false, false);
            v[q] = __builtin_bit_cast(float, (uint32_t)h[0]) + __builtin_bit_cast(float, (uint32_t)h[1]);
        }
        if constexpr (G >= 64) {
            const auto h = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v[q]),
                                                            __builtin_bit_cast(uint32_t, v[q]), false, false);
            v[q] = __builtin_bit_cast(float, (uint32_t)h[0]) + __builtin_bit_cast(float, (uint32_t)h[1]);
        }
    }
    if constexpr (G > 64) {
        constexpr int kWaves = norm_threads(G) / 64, kOfRow = G / 64;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int q = 0; q < N; ++q) slots[q * kWaves + wave] = v[q];
        }
        __syncthreads();
        const int first = wave / kOfRow * kOfRow;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            v[q] = slots[q * kWaves + first];
#pragma unroll
            for (int w = 1; w < kOfRow; ++w) v[q] += slots[q * kWaves + first + w];
        }
    }
}

// 1 / sqrt(v) for v of eps (a normal number) or more: the instruction's value (off by
// 2^-23 at most) and a Newton step, 8 instructions where the library's root and
// division take 40.
__device__ __forceinline__ float reciprocal_root(float v) {
    const float r = __builtin_amdgcn_rsqf(v);
    return fmaf(0.5f * r, fmaf(-(v * r), r, 1.f), r);
}

// The normalised row is f r + c: f the deviations from the mean in place (0 past d),
// r = 1 / sqrt(variance + eps).  The sum's mean is off by some 2^-20 of the
// entries' size, in every deviation alike; so they have that for their mean, which
// c takes off them.  (A variance of 2^-20 of that squared is no more than the
// roundings of the two: what is less, for a row of one value, counts as that.)
template <int G>
__device__ __forceinline__ void statistics(float (&f)[8], int k, int d, float eps, float (*slots)[16], float &r, float &c) {
    const float each = 1.f / (float)d;
    float s[1] = {((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]))};
    row_sums<G, 1>(s, slots[0]);
    const float m = s[0] * each, m0 = k < d ? m : 0.f, m1 = k + 4 < d ? m : 0.f;   // (entries past d are 0)
    float two[2] = {0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 8; ++q) f[q] -= q < 4 ? m0 : m1;
    two[0] = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
#pragma unroll
    for (int q = 0; q < 8; ++q) two[1] = fmaf(f[q], f[q], two[1]);
    row_sums<G, 2>(two, slots[1]);
    const float rest = two[0] * each, v = fmaf(-rest, rest, two[1] * each), least = rest * rest * 0x1p-20f;
    r = reciprocal_root((v < least ? least : v) + eps);   // (a NaN stays one)
    c = -rest * r;
}

// A lane's entries of gamma or beta (`none` where there is no array).
__device__ __forceinline__ void weights(const float *p, int k, int d, float none, float (&f)[8]) {
    Raw<float> raw;
    if (p != nullptr) raw.load(p, k, d);
    raw.widen(f);
#pragma unroll
    for (int q = 0; q < 8; ++q) f[q] = p != nullptr ? f[q] : none;
}

// A workgroup's chunks of the rows, a row for each of its groups of lanes: the
// next chunk's is on its way while one is worked on, and the id of the one after
// it.
template <int G>
struct Ahead {
    const int32_t *posts;
    int chunks, id, id1, id2;
    __device__ __forceinline__ int id_of(int chunk) const {
        constexpr int kRows = norm_threads(G) / G, kChunks = kBiaRows / kRows;
        static_assert(kBiaRows % kRows == 0, "a block of posts is a whole number of chunks");
        const int c = min(chunk, chunks - 1);
        const int v = posts[(size_t)(c / kChunks) * kPostRec + c % kChunks * kRows + threadIdx.x / G];
        return chunk < chunks ? v : -1;
    }
    __device__ __forceinline__ Ahead(const int32_t *posts, int chunks) : posts(posts), chunks(chunks) {
        id1 = id_of(blockIdx.x);
        id2 = id_of(blockIdx.x + gridDim.x);
    }
    __device__ __forceinline__ void take() { id = id1, id1 = id2; }
};

template <typename T, int G>
__global__ __launch_bounds__(norm_threads(G)) void norm_kernel(const int32_t *__restrict__ posts, int chunks, int d,
                                                               const T *__restrict__ x, const float *__restrict__ gamma,
                                                               const float *__restrict__ beta, float eps,
                                                               uint16_t *__restrict__ y) {
    __shared__ float slots[3][16];
    const int k = 8 * (threadIdx.x & (G - 1));
    Ahead<G> rows(posts, chunks);
    Raw<T> raw;
    auto load = [&]() {
        raw = Raw<T>();
        if (rows.id1 >= 0) raw.load(x + (size_t)rows.id1 * d, k, d);
    };
    load();
    float g[8], b[8];
    weights(gamma, k, d, 1.f, g);
    weights(beta, k, d, 0.f, b);
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        float f[8];
        raw.widen(f);
        rows.take();
        load();
        rows.id2 = rows.id_of(c + 2 * gridDim.x);
        float r, rest;
        statistics<G>(f, k, d, eps, slots, r, rest);
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] = fmaf(fmaf(f[q], r, rest), g[q], b[q]);
        if (rows.id >= 0) store(y + (size_t)rows.id * d, k, d, f);
    }
}

// dx, and a workgroup's share of dgamma and dbeta (PARTS; [2][8 G] floats each,
// or the results themselves where there is one workgroup).
template <typename T, int G, bool PARTS>
__global__ __launch_bounds__(norm_threads(G)) void norm_bwd_kernel(const int32_t *__restrict__ posts, int chunks, int d,
                                                                   const T *__restrict__ x,
                                                                   const float *__restrict__ gamma,
                                                                   const uint16_t *__restrict__ dy, float eps,
                                                                   T *__restrict__ dx, float *__restrict__ parts,
                                                                   float *__restrict__ dgamma, float *__restrict__ dbeta) {
    constexpr int kRows = norm_threads(G) / G;
    __shared__ float slots[3][16], slots2[2 * 16];
    __shared__ float sums[PARTS && kRows > 1 ? kRows * 16 * G : 1];
    const int k = 8 * (threadIdx.x & (G - 1));
    const float each = 1.f / (float)d;
    float g[8], sg[8], sb[8];
    weights(gamma, k, d, 1.f, g);
#pragma unroll
    for (int q = 0; q < 8; ++q) sg[q] = sb[q] = 0.f;
    Ahead<G> rows(posts, chunks);
    Raw<T> raw;
    Raw<uint16_t> up;
    auto load = [&]() {
        raw = Raw<T>();
        up = Raw<uint16_t>();
        if (rows.id1 >= 0) {
            raw.load(x + (size_t)rows.id1 * d, k, d);
            up.load(dy + (size_t)rows.id1 * d, k, d);
        }
    };
    load();
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        float f[8], e[8], two[2] = {0.f, 0.f};
        raw.widen(f);
        up.widen(e);
        rows.take();
        load();
        rows.id2 = rows.id_of(c + 2 * gridDim.x);
        float r, rest;
        statistics<G>(f, k, d, eps, slots, r, rest);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            f[q] = fmaf(f[q], r, rest);   // (past d the gradient is 0)
            if constexpr (PARTS) {   // (a row that is not there adds zeros)
                sg[q] = fmaf(e[q], f[q], sg[q]);
                sb[q] += e[q];
            }
            e[q] *= g[q];
            two[0] += e[q];
            two[1] = fmaf(e[q], f[q], two[1]);
        }
        row_sums<G, 2>(two, slots2);
        const float s = -r * (two[0] * each), t = -r * (two[1] * each);
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] = fmaf(f[q], t, fmaf(e[q], r, s));
        if (dx != nullptr && rows.id >= 0) store(dx + (size_t)rows.id * d, k, d, f);
    }
    if constexpr (PARTS) {
        if constexpr (kRows > 1) {
            float *own = sums + (threadIdx.x / G) * 16 * G;
#pragma unroll
            for (int q = 0; q < 8; ++q) own[k + q] = sg[q], own[8 * G + k + q] = sb[q];
            __syncthreads();
            for (int c = threadIdx.x; c < 16 * G; c += norm_threads(G)) {
                float s = sums[c];
                for (int w = 1; w < kRows; ++w) s += sums[w * 16 * G + c];
                if (gridDim.x > 1) {
                    parts[(size_t)blockIdx.x * 16 * G + c] = s;
                } else {
                    const int a = c & (8 * G - 1);
                    float *out = c < 8 * G ? dgamma : dbeta;
                    if (a < d && out != nullptr) out[a] = s;
                }
            }
        } else if (gridDim.x > 1) {
            float *own = parts + (size_t)blockIdx.x * 16 * G;
#pragma unroll
            for (int q = 0; q < 8; ++q) own[k + q] = sg[q], own[8 * G + k + q] = sb[q];
        } else {
            if (dgamma != nullptr) store(dgamma, k, d, sg);
            if (dbeta != nullptr) store(dbeta, k, d, sb);
        }
    }
}

// The shares of dgamma and dbeta added up in a fixed order: a workgroup takes
// 32 columns, thread (c, p) every 32nd share.  (4.3 us of 650 shares of 1,024
// floats, 2.5 of them the launch.)
constexpr int kJoinCols = 32, kJoinLanes = 32;
__global__ __launch_bounds__(kJoinCols *kJoinLanes) void norm_join_kernel(const float *__restrict__ parts, int count,
                                                                          int wide, int d, float *__restrict__ dgamma,
                                                                          float *__restrict__ dbeta) {
    __shared__ float part[kJoinLanes][kJoinCols + 1];
    const int c = threadIdx.x % kJoinCols, p = threadIdx.x / kJoinCols, at = blockIdx.x * kJoinCols + c;
    float s = 0.f;
#pragma unroll 8
    for (int q = p; q < count; q += kJoinLanes) s += parts[(size_t)q * 2 * wide + at];
    part[p][c] = s;
    __syncthreads();
    for (int half = kJoinLanes / 2; half > 0; half /= 2) {
        if (p < half) part[p][c] += part[p + half][c];
        __syncthreads();
    }
    if (p == 0) {
        const int a = at < wide ? at : at - wide;
        float *out = at < wide ? dgamma : dbeta;
        if (a < d && out != nullptr) out[a] = part[0][c];
    }
}

// Lanes a row of d entries takes: 16, 32 ... 1024.
int norm_lanes(int d) {
    int g = 16;
    while (8 * g < d) g *= 2;
    return g;
}
int norm_chunks(const KernelPlan &p, int G) { return p.n_posts * (kBiaRows / (norm_threads(G) / G)); }
// Workgroups that share the sums: two chunks each at least, where there are many
// (200 sentences of d = 500: 15.4 us with one, 14.5 with two, 15.6 with three).
int norm_parts(const KernelPlan &p, int G) {
    const int chunks = norm_chunks(p, G), most = (G > 64 ? kNormMostBwdWide : kNormMostBwd) * 256 / norm_threads(G);
    return std::min(std::max(std::min(chunks, 512), chunks / 2), most);
}

template <typename T, int G>
void launch_norm_g(const KernelPlan &p, const void *x, int d, const float *gamma, const float *beta, float eps, uint16_t *y,
                   hipStream_t stream) {
    const int chunks = norm_chunks(p, G);
    hipLaunchKernelGGL((norm_kernel<T, G>), dim3(std::min(chunks, kNormMost * 256 / norm_threads(G))), dim3(norm_threads(G)),
                       0, stream, p.posts, chunks, d, static_cast<const T *>(x), gamma, beta, eps, y);
}

template <typename T, int G>
void launch_norm_bwd_g(const KernelPlan &p, const void *x, int d, const float *gamma, const uint16_t *dy, float eps,
                       void *dx, float *dgamma, float *dbeta, float *parts, hipStream_t stream) {
    const int chunks = norm_chunks(p, G), count = norm_parts(p, G);
    if (dgamma == nullptr && dbeta == nullptr) {
        hipLaunchKernelGGL((norm_bwd_kernel<T, G, false>), dim3(std::min(chunks, kNormMost * 256 / norm_threads(G))),
                           dim3(norm_threads(G)), 0, stream, p.posts, chunks, d, static_cast<const T *>(x), gamma, dy, eps,
                           static_cast<T *>(dx), nullptr, nullptr, nullptr);
        return;
    }
    hipLaunchKernelGGL((norm_bwd_kernel<T, G, true>), dim3(count), dim3(norm_threads(G)), 0, stream, p.posts, chunks, d,
                       static_cast<const T *>(x), gamma, dy, eps, static_cast<T *>(dx), parts, dgamma, dbeta);
    if (count > 1)
        hipLaunchKernelGGL(norm_join_kernel, dim3(16 * G / kJoinCols), dim3(kJoinCols * kJoinLanes), 0, stream, parts, count,
                           8 * G, d, dgamma, dbeta);
}

#define CRF_NORM_LANES(T, CALL, ...)                   \
    switch (norm_lanes(d)) {                           \
        case 16: CALL<T, 16>(__VA_ARGS__); break;      \
        case 32: CALL<T, 32>(__VA_ARGS__); break;      \
        case 64: CALL<T, 64>(__VA_ARGS__); break;      \
        case 128: CALL<T, 128>(__VA_ARGS__); break;    \
        case 256: CALL<T, 256>(__VA_ARGS__); break;    \
        case 512: CALL<T, 512>(__VA_ARGS__); break;    \
        default: CALL<T, 1024>(__VA_ARGS__); break;    \
    }

}  // namespace

int64_t norm_bwd_bytes(const KernelPlan &p, int d) {
    const int G = norm_lanes(d);
    return ((int64_t)norm_parts(p, G) * 16 * G * 4 + 255) / 256 * 256;
}

hipError_t launch_norm(const KernelPlan &p, const void *x, bool f32, int d, const float *gamma, const float *beta,
                       float eps, uint16_t *y, hipStream_t stream) {
    if (f32)
        CRF_NORM_LANES(float, launch_norm_g, p, x, d, gamma, beta, eps, y, stream)
    else
        CRF_NORM_LANES(uint16_t, launch_norm_g, p, x, d, gamma, beta, eps, y, stream)
    return hipGetLastError();
}

hipError_t launch_norm_bwd(const KernelPlan &p, const void *x, bool f32, int d, const float *gamma, const uint16_t *dy,
                           float eps, void *dx, float *dgamma, float *dbeta, char *ws, hipStream_t stream) {
    float *parts = reinterpret_cast<float *>(ws);
    if (f32)
        CRF_NORM_LANES(float, launch_norm_bwd_g, p, x, d, gamma, dy, eps, dx, dgamma, dbeta, parts, stream)
    else
        CRF_NORM_LANES(uint16_t, launch_norm_bwd_g, p, x, d, gamma, dy, eps, dx, dgamma, dbeta, parts, stream)
    return hipGetLastError();
}

}  // namespace crf
