// crf_ortho.hip -- a matrix's nearest orthogonal one by Newton-Schulz products,
// and the update of weights by their orthogonalised momentum.
//
// With U the matrix (p rows, q >= p columns; a taller one is taken transposed),
//     X = U / (|U|_F + eps), and for each of the steps' (a, b, c):
//     A = X X^T,   B = b A + c A A,   X <- a X + B X,
// which keeps U's singular vectors and takes each singular value s to
// a s + b s^3 + c s^5, step by step towards 1.
//
// Products on the matrix cores.  A step multiplies what earlier ones have left
// of the small singular values by a (3.4 with the usual coefficients, 480 over
// five steps), so operands of 8 or 11 bits do not do.  Every matrix is held
// as two float16 parts, x = hi + lo (22 bits), and a product takes
// hi hi + hi lo + lo hi with float32 sums (lo lo, 2^-22 of the product, is left
// out): three float16 products at 16 times the float32 rate each.  Parts of
// values below float16's normal range lose digits, so X, A and B are held
// scaled by powers of two that leave room for what the caller's coefficients
// let the entries grow to, and no more.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "crf_internal.h"

namespace crf {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 64;             // rows and columns of an output tile
constexpr int kStepK = 64;            // K staged at a time
constexpr int kKStride = kStepK + 8;  // row stride of a staged piece
constexpr int kNormChunk = 8192;      // entries of a share of a matrix's norm

// What X, A and B are held times: entries of at most 8, 32 and 64 fit float16.
constexpr float kScaleX = 4096.f, kScaleA = 2048.f, kScaleB = 1024.f;

// One matrix's arrays, each two planes (hi, then lo) of float16.
struct OrthoShape {
    int p, q;          // sides, p <= q
    int pp, qq;        // padded to whole tiles
    __host__ __device__ int64_t x_plane() const { return (int64_t)pp * qq; }
    __host__ __device__ int64_t a_plane() const { return (int64_t)pp * pp; }
};
__host__ __device__ inline OrthoShape ortho_shape(int rows, int cols) {
    OrthoShape s;
    s.p = rows < cols ? rows : cols;
    s.q = rows < cols ? cols : rows;
    s.pp = (s.p + kTile - 1) / kTile * kTile;
    s.qq = (s.q + kTile - 1) / kTile * kTile;
    return s;
}
inline int norm_shares(int rows, int cols) { return (int)(((int64_t)rows * cols + kNormChunk - 1) / kNormChunk); }

// The caller's matrices.
struct OrthoIo {
    const float *grad, *momentum, *w;   // momentum NULL: U is grad itself
    float *momentum_out, *out;          // out: X, or the new weights where w is given
    int rows, cols, ld;
    float mu;
    int nesterov;
    float keep, rate, eps;              // out = keep w - rate X
};

__device__ __forceinline__ float updated(const OrthoIo &io, float g, float m) {
    return io.nesterov ? fmaf(io.mu, m, g) : m;
}

// The new momentum, and shares of each matrix's sum of squares of U in 64 bits
// (squares of float32 values neither overflow there nor vanish).
__global__ __launch_bounds__(256) void ortho_norm_kernel(OrthoIo io, double *__restrict__ shares) {
    __shared__ double part[256];
    const int64_t size = (int64_t)io.rows * io.ld, first = (int64_t)blockIdx.x * kNormChunk;
    const int64_t base = blockIdx.y * size, count = (int64_t)io.rows * io.cols;
    double s = 0.0;
    for (int64_t k = first + threadIdx.x; k < min(first + kNormChunk, count); k += 256) {
        const int64_t row = k / io.cols, at = base + row * io.ld + (k - row * io.cols);
        float u = io.grad[at];
        if (io.momentum != nullptr) {
            const float m = fmaf(io.mu, io.momentum[at], u);
            io.momentum_out[at] = m;
            u = updated(io, u, m);
        }
        s += (double)u * (double)u;
    }
    part[threadIdx.x] = s;
    __syncthreads();
    for (int half = 128; half > 0; half /= 2) {
        if (threadIdx.x < half) part[threadIdx.x] += part[threadIdx.x + half];
        __syncthreads();
    }
    if (threadIdx.x == 0) shares[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = part[0];
}

__device__ __forceinline__ void split(float v, _Float16 &hi, _Float16 &lo) {
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// X = U / (|U|_F + eps) in parts, and its transpose; zeros past the matrix.
__global__ __launch_bounds__(256) void ortho_load_kernel(OrthoIo io, const double *__restrict__ shares, int n_shares,
                                                         _Float16 *__restrict__ x, _Float16 *__restrict__ xt) {
    __shared__ float tile[kTile][kTile + 1];
    __shared__ double total;
    const OrthoShape sh = ortho_shape(io.rows, io.cols);
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int k = 0; k < n_shares; ++k) s += shares[(int64_t)blockIdx.z * n_shares + k];
        total = s;
    }
    __syncthreads();
    // (a sum that is not finite makes the whole matrix NaN)
    const double inv = (double)kScaleX / (sqrt(total) + (double)io.eps) + 0.0 * total;
    const bool tall = io.rows > io.cols;
    const int i0 = blockIdx.y * kTile, j0 = blockIdx.x * kTile;   // of X
    const int64_t base = (int64_t)blockIdx.z * io.rows * io.ld;
    for (int t = threadIdx.x; t < kTile * kTile; t += 256) {
        const int r = t / kTile, c = t % kTile;   // along the caller's rows
        const int row = (tall ? j0 : i0) + r, col = (tall ? i0 : j0) + c;
        float u = 0.f;
        if (row < io.rows && col < io.cols) {
            const int64_t at = base + (int64_t)row * io.ld + col;
            u = io.grad[at];
            if (io.momentum != nullptr) u = updated(io, u, io.momentum_out[at]);
            u = (float)((double)u * inv);
        }
        tile[tall ? c : r][tall ? r : c] = u;
    }
    __syncthreads();
    x += blockIdx.z * 2 * sh.x_plane();
    xt += blockIdx.z * 2 * sh.x_plane();
    for (int t = threadIdx.x; t < kTile * kTile; t += 256) {
        const int r = t / kTile, c = t % kTile;
        _Float16 hi, lo;
        split(tile[r][c], hi, lo);
        const int64_t at = (int64_t)(i0 + r) * sh.qq + j0 + c;
        x[at] = hi;
        x[sh.x_plane() + at] = lo;
        split(tile[c][r], hi, lo);
        const int64_t tat = (int64_t)(j0 + r) * sh.pp + i0 + c;
        xt[tat] = hi;
        xt[sh.x_plane() + tat] = lo;
    }
}

enum Product { kGram, kPoly, kNext, kLast };

// One tile of a product of two matrices whose rows run along K:
//   kGram  A = X X^T;             kPoly  B = b A + c A A;
//   kNext  X' = a X + B X (from B and X^T), and its transpose;   kLast  the same, to the caller.
struct ProductArgs {
    const _Float16 *left, *right;   // operands
    const _Float16 *add;            // A for kPoly, X for kNext and kLast
    _Float16 *out, *out_t;
    int k, add_stride;              // K; row stride of add and out
    int64_t left_plane, right_plane, add_plane;
    float a, c;                     // out = a add + c product, in the scales of the result
    int t_stride;
};

__device__ __forceinline__ f16x8 frag(const _Float16 *p) { return *reinterpret_cast<const f16x8 *>(p); }

template <int KIND>
__global__ __launch_bounds__(256) void ortho_product_kernel(ProductArgs g, OrthoIo io) {
    __shared__ __align__(16) _Float16 stage[4][kTile][kKStride];   // left hi, lo, right hi, lo
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int i0 = blockIdx.y * kTile, j0 = blockIdx.x * kTile;
    const _Float16 *left = g.left + blockIdx.z * 2 * g.left_plane + (int64_t)i0 * g.k;
    const _Float16 *right = g.right + blockIdx.z * 2 * g.right_plane + (int64_t)j0 * g.k;
    // thread t stages rows t / 8 and t / 8 + 32, entries 8 (t % 8) .. + 7
    const int sr = tid >> 3, sk = 8 * (tid & 7);
    u32x4 next[4][2];
    auto load = [&](int k0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = (int64_t)(sr + 32 * h) * g.k + k0 + sk;
            next[0][h] = *reinterpret_cast<const u32x4 *>(left + at);
            next[1][h] = *reinterpret_cast<const u32x4 *>(left + g.left_plane + at);
            next[2][h] = *reinterpret_cast<const u32x4 *>(right + at);
            next[3][h] = *reinterpret_cast<const u32x4 *>(right + g.right_plane + at);
        }
    };
    load(0);
    f32x4 acc[2][2];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int wi = 32 * (wave >> 1), wj = 32 * (wave & 1);   // the wavefront's part of the tile
    for (int k0 = 0; k0 < g.k; k0 += kStepK) {
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) *reinterpret_cast<u32x4 *>(&stage[s][sr + 32 * h][sk]) = next[s][h];
        __syncthreads();
        if (k0 + kStepK < g.k) load(k0 + kStepK);
#pragma unroll
        for (int k = 0; k < kStepK; k += 32) {
            f16x8 l[2][2], r[2][2];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    l[s][m] = frag(&stage[s][wi + 16 * m + (lane & 15)][k + 8 * (lane >> 4)]);
                    r[s][m] = frag(&stage[2 + s][wj + 16 * m + (lane & 15)][k + 8 * (lane >> 4)]);
                }
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(l[0][m], r[1][n], acc[m][n], 0, 0, 0);
                    acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(l[1][m], r[0][n], acc[m][n], 0, 0, 0);
                    acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(l[0][m], r[0][n], acc[m][n], 0, 0, 0);
                }
        }
    }
    // a lane holds rows 4 (lane / 16) .. + 3 of column lane % 16
    const OrthoShape sh = ortho_shape(io.rows, io.cols);
    const bool tall = io.rows > io.cols;
    const _Float16 *add = KIND == kGram ? nullptr : g.add + blockIdx.z * 2 * g.add_plane;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int i = i0 + wi + 16 * m + 4 * (lane >> 4), j = j0 + wj + 16 * n + (lane & 15);
            f16x4 hi, lo;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int64_t at = (int64_t)(i + t) * g.add_stride + j;
                float v = g.c * acc[m][n][t];
                if constexpr (KIND != kGram) v = fmaf(g.a, (float)add[at] + (float)add[g.add_plane + at], v);
                if constexpr (KIND == kLast) {
                    if (i + t < sh.p && j < sh.q) {
                        const int64_t to = (int64_t)blockIdx.z * io.rows * io.ld +
                                           (tall ? (int64_t)j * io.ld + i + t : (int64_t)(i + t) * io.ld + j);
                        io.out[to] = io.w != nullptr ? fmaf(-io.rate, v, io.keep * io.w[to]) : v;
                    }
                } else {
                    _Float16 a, b;
                    split(v, a, b);
                    hi[t] = a;
                    lo[t] = b;
                    _Float16 *out = g.out + blockIdx.z * 2 * g.add_plane;
                    out[at] = a;
                    out[g.add_plane + at] = b;
                }
            }
            if constexpr (KIND == kNext) {
                _Float16 *out = g.out_t + blockIdx.z * 2 * g.add_plane + (int64_t)j * g.t_stride + i;
                *reinterpret_cast<f16x4 *>(out) = hi;
                *reinterpret_cast<f16x4 *>(out + g.add_plane) = lo;
            }
        }
}

int64_t aligned(int64_t n) { return (n + 255) / 256 * 256; }

}  // namespace

int64_t ortho_bytes(int count, int rows, int cols) {
    const OrthoShape sh = ortho_shape(rows, cols);
    return aligned(8 * (int64_t)count * norm_shares(rows, cols)) + 4 * aligned(4 * count * sh.x_plane()) +
           2 * aligned(4 * count * sh.a_plane());
}

hipError_t launch_ortho(const float *grad, const float *momentum, const float *w, float *momentum_out, float *out, int count,
                        int rows, int cols, int ld, float mu, bool nesterov, float keep, float rate, float eps,
                        const float *coefficients, int steps, char *ws, hipStream_t stream) {
    const OrthoShape sh = ortho_shape(rows, cols);
    OrthoIo io{grad, momentum, w, momentum_out, out, rows, cols, ld, mu, nesterov, keep, rate, eps};
    double *shares = reinterpret_cast<double *>(ws);
    ws += aligned(8 * (int64_t)count * norm_shares(rows, cols));
    _Float16 *x[2], *xt[2], *a, *b;
    auto take = [&](int64_t plane) {
        _Float16 *at = reinterpret_cast<_Float16 *>(ws);
        ws += aligned(4 * count * plane);
        return at;
    };
    for (int k = 0; k < 2; ++k) x[k] = take(sh.x_plane()), xt[k] = take(sh.x_plane());
    a = take(sh.a_plane());
    b = take(sh.a_plane());
    const int n_shares = norm_shares(rows, cols), tp = sh.pp / kTile, tq = sh.qq / kTile;
    hipLaunchKernelGGL(ortho_norm_kernel, dim3(n_shares, count), dim3(256), 0, stream, io, shares);
    hipLaunchKernelGGL(ortho_load_kernel, dim3(tq, tp, count), dim3(256), 0, stream, io, shares, n_shares, x[0], xt[0]);
    for (int s = 0; s < steps; ++s) {
        const float *co = coefficients + 3 * s;
        const int now = s & 1;
        const ProductArgs gram{x[now], x[now], nullptr, a, nullptr, sh.qq, sh.pp, sh.x_plane(), sh.x_plane(), sh.a_plane(),
                               0.f, kScaleA / (kScaleX * kScaleX), 0};
        const ProductArgs poly{a, a, a, b, nullptr, sh.pp, sh.pp, sh.a_plane(), sh.a_plane(), sh.a_plane(),
                               co[1] * (kScaleB / kScaleA), co[2] * (kScaleB / (kScaleA * kScaleA)), 0};
        hipLaunchKernelGGL(ortho_product_kernel<kGram>, dim3(tp, tp, count), dim3(256), 0, stream, gram, io);
        hipLaunchKernelGGL(ortho_product_kernel<kPoly>, dim3(tp, tp, count), dim3(256), 0, stream, poly, io);
        const bool last = s + 1 == steps;
        const float to = last ? 1.f : kScaleX;
        const ProductArgs next{b, xt[now], x[now], x[now ^ 1], xt[now ^ 1], sh.pp, sh.qq, sh.a_plane(), sh.x_plane(),
                               sh.x_plane(), co[0] * (to / kScaleX), to / (kScaleB * kScaleX), sh.pp};
        if (last)
            hipLaunchKernelGGL(ortho_product_kernel<kLast>, dim3(tq, tp, count), dim3(256), 0, stream, next, io);
        else
            hipLaunchKernelGGL(ortho_product_kernel<kNext>, dim3(tq, tp, count), dim3(256), 0, stream, next, io);
    }
    return hipGetLastError();
}

}  // namespace crf
