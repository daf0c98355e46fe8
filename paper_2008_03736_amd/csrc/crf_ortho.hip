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

#include "../../include/crf_inside.h"
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

__device__ __forceinline__ void split(const f32x4 &v, f16x4 &hi, f16x4 &lo) {
    hi = __builtin_convertvector(v, f16x4);
    lo = __builtin_convertvector(v - __builtin_convertvector(hi, f32x4), f16x4);
}
__device__ __forceinline__ f32x4 joined(const f16x4 &hi, const f16x4 &lo) {
    return __builtin_convertvector(hi, f32x4) + __builtin_convertvector(lo, f32x4);
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

// Matrices of up to kSmall x kSmall: a workgroup of W wavefronts each, which never
// leaves its CU.  Wavefront w owns X's columns 16 w .. + 15, in registers.  Their
// parts are wanted twice over: in LDS, as rows of X, for the Gram matrix, and in
// the owner's registers as the right operand of B X -- a product's result has, a
// lane, four consecutive rows of one column, and two tiles of it are just a right
// operand's fragment whose K runs 0-3, 16-19 | 4-7, 20-23 | ...; the Gram matrix
// and B are stored with their columns in that order, so that no product minds.
// A and B are symmetric: of the tiles (i, j) and (j, i) one is computed, column
// j taking rows j, j + 1 .. j + PT / 2 (cyclically), which shares the work
// evenly.
constexpr int kSmall = 128;
__host__ __device__ constexpr int small_stride(int tiles) { return (tiles + 1) / 2 * 32 + 8; }   // of a row of 16 `tiles`
inline int64_t small_lds(int p, int q) {
    const int pt = (p + 15) / 16, qt = (q + 15) / 16;
    const int64_t parts = 2 * 2 * 16 * pt * (int64_t)(small_stride(pt) + small_stride(qt));
    return std::max<int64_t>(parts, 4 * (int64_t)q * (p + 1));
}

struct Steps {
    float f[CRF_MAX_STEPS][3];
    int count;
};

// U row tiles of a stored matrix (hi, and lo `plane` entries on) times a column
// tile in registers: tile u is at row tile row(u), and done(u, acc) takes its
// result.  ks: steps of K.  The next tile's fragments fly while this one's
// products run, in a chain for each of the three.
template <int U, int KS, typename Row, typename Done>
__device__ __forceinline__ void row_tiles(const _Float16 *from, int plane, int stride, int ks, const f16x8 (&rh)[KS],
                                          const f16x8 (&rl)[KS], Row row, Done done) {
    f16x8 lh[2][KS], ll[2][KS];
    auto load = [&](int u) {
        const _Float16 *at = from + 16 * row(u) * stride;
#pragma unroll
        for (int s = 0; s < KS; ++s)
            if (s < ks) {
                lh[u & 1][s] = frag(at + 32 * s);
                ll[u & 1][s] = frag(at + plane + 32 * s);
            }
    };
    load(0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (u + 1 < U) load(u + 1);
        f32x4 acc[3];
#pragma unroll
        for (int t = 0; t < 3; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s)
            if (s < ks) {
                acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lh[u & 1][s], rl[s], acc[0], 0, 0, 0);
                acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ll[u & 1][s], rh[s], acc[1], 0, 0, 0);
                acc[2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lh[u & 1][s], rh[s], acc[2], 0, 0, 0);
            }
        done(u, (acc[0] + acc[1]) + acc[2]);
        __builtin_amdgcn_sched_barrier(0);   // (no further loads ahead: their registers spill)
    }
}

template <int PT, int W>
__global__ __launch_bounds__(64 * W) void ortho_small_kernel(OrthoIo io, Steps steps) {
    constexpr int kKP = (PT + 1) / 2;   // steps of K over p
    constexpr int kKQ = W / 2;          // most steps of K over q
    constexpr int kT = PT / 2 + 1;      // row tiles of a column of A and B
    constexpr int kSG = small_stride(PT);
    constexpr int kThreads = 64 * W;
    extern __shared__ __align__(16) char smem[];
    __shared__ double norm[W];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int n = lane & 15, g = lane >> 4;
    const bool tall = io.rows > io.cols;
    const int p = tall ? io.cols : io.rows, q = tall ? io.rows : io.cols;
    const int qt = (q + 15) / 16, kq = (qt + 1) / 2, sx = small_stride(qt);
    _Float16 *xs = reinterpret_cast<_Float16 *>(smem), *gs = xs + 2 * 16 * PT * sx;
    const int x_plane = 16 * PT * sx;
    constexpr int g_plane = 16 * PT * kSG;
    const int64_t base = (int64_t)blockIdx.x * io.rows * io.ld;

    // U, the new momentum and the norm
    float *us = reinterpret_cast<float *>(smem);
    const int us_stride = io.cols + 1;
    double sum = 0.0;
    int row = tid / io.cols, col = tid - row * io.cols;   // of entry tid, tid + kThreads ..
    const int down = kThreads / io.cols, right = kThreads - down * io.cols;
    constexpr int kAhead = 10;   // entries in flight
    while (row < io.rows) {
        float u[kAhead], m[kAhead];
        int r[kAhead], c[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            r[e] = row;
            c[e] = col;
            const int64_t at = base + (int64_t)min(row, io.rows - 1) * io.ld + col;
            u[e] = io.grad[at];
            if (io.momentum != nullptr) m[e] = io.momentum[at];
            col += right;
            row += down;
            if (col >= io.cols) col -= io.cols, ++row;
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
            if (r[e] < io.rows) {
                if (io.momentum != nullptr) {
                    m[e] = fmaf(io.mu, m[e], u[e]);
                    io.momentum_out[base + (int64_t)r[e] * io.ld + c[e]] = m[e];
                    u[e] = updated(io, u[e], m[e]);
                }
                us[r[e] * us_stride + c[e]] = u[e];
                sum += (double)u[e] * (double)u[e];
            }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
    if (lane == 0) norm[wave] = sum;
    __syncthreads();
    sum = norm[0];
#pragma unroll
    for (int w = 1; w < W; ++w) sum += norm[w];
    // (a sum that is not finite makes the whole matrix NaN)
    const double inv = 1.0 / (sqrt(sum) + (double)io.eps) + 0.0 * sum;
    // tile i: rows 16 i + 4 g .. + 3 of column own
    f32x4 x[PT];
    const int own = 16 * wave + n;
#pragma unroll
    for (int i = 0; i < PT; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int r = 16 * i + 4 * g + t, row = min(r, p - 1), at = min(own, q - 1);
            const float u = (float)((double)us[tall ? at * us_stride + row : row * us_stride + at] * inv);
            x[i][t] = r < p && own < q ? u : 0.f;
        }
    __syncthreads();
    for (int k = tid; k < (2 * x_plane + 2 * g_plane) / 8; k += kThreads) reinterpret_cast<u32x4 *>(xs)[k] = u32x4{0u, 0u, 0u, 0u};
    __syncthreads();

#pragma unroll 1
    for (int step = 0; step < steps.count; ++step) {
        const float a = steps.f[step][0], b = steps.f[step][1], c3 = steps.f[step][2];
        // (a step's LDS addresses are taken from these anew: kept over the loop,
        // some hundred of them, they would take the registers that X lies in)
        asm("" : "+v"(n), "+v"(g));
        // X's parts: the owner's columns into the rows in LDS, and kept as fragments
        f16x8 xh[kKP], xl[kKP];
#pragma unroll
        for (int i = 0; i < 2 * kKP; ++i) {
            f16x4 hi = f16x4{0, 0, 0, 0}, lo = hi;
            if (i < PT) {
                split(kScaleX * x[i < PT ? i : 0], hi, lo);
                if (wave < qt) {
                    _Float16 *to = xs + (16 * i + 4 * g) * sx + 16 * wave + n;
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        to[t * sx] = hi[t];
                        to[x_plane + t * sx] = lo[t];
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                xh[i >> 1][4 * (i & 1) + t] = hi[t];
                xl[i >> 1][4 * (i & 1) + t] = lo[t];
            }
        }
        __syncthreads();

        // Symmetric products: column tile j, row tiles j + u (cyclically)
        const int j = wave;
        auto row_tile = [&](int u) { return j + u < PT ? j + u : j + u - PT; };
        auto wanted = [&](int u) { return PT % 2 != 0 || u < PT / 2 || j < PT / 2; };
        // where tile (i, j)'s lane puts its four rows: row 16 j + n of the stored
        // matrix, columns 16 i + 4 g .. + 3 in their order, and the mirror image
        auto place = [&](int i) { return (16 * j + n) * kSG + 32 * (i >> 1) + 8 * g + 4 * (i & 1); };
        auto put = [&](int u, const f32x4 &v) {
            const int i = row_tile(u);
            f16x4 hi, lo;
            split(v, hi, lo);
            *reinterpret_cast<f16x4 *>(gs + place(i)) = hi;
            *reinterpret_cast<f16x4 *>(gs + g_plane + place(i)) = lo;
            if (u > 0) {
                const int at = (16 * i + 4 * g) * kSG + 32 * (j >> 1) + 8 * (n >> 2) + 4 * (j & 1) + (n & 3);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    gs[at + t * kSG] = hi[t];
                    gs[g_plane + at + t * kSG] = lo[t];
                }
            }
        };

        // A = X X^T
        if (j < PT) {
            f16x8 rh[kKQ], rl[kKQ];
#pragma unroll
            for (int s = 0; s < kKQ; ++s)
                if (s < kq) {
                    const _Float16 *from = xs + (16 * j + n) * sx + 32 * s + 8 * g;
                    rh[s] = frag(from);
                    rl[s] = frag(from + x_plane);
                }
            row_tiles<kT>(xs + n * sx + 8 * g, x_plane, sx, kq, rh, rl, row_tile, [&](int u, const f32x4 &acc) {
                if (wanted(u)) put(u, acc * (kScaleA / (kScaleX * kScaleX)));
            });
        }
        __syncthreads();

        // B = b A + c A A, held until every wavefront has read A
        f32x4 poly[kT];
        if (j < PT) {
            f16x8 rh[kKP], rl[kKP];
#pragma unroll
            for (int s = 0; s < kKP; ++s) {
                const _Float16 *from = gs + (16 * j + n) * kSG + 32 * s + 8 * g;
                rh[s] = frag(from);
                rl[s] = frag(from + g_plane);
            }
            row_tiles<kT>(gs + n * kSG + 8 * g, g_plane, kSG, kKP, rh, rl, row_tile, [&](int u, const f32x4 &acc) {
                const f16x4 hi = *reinterpret_cast<const f16x4 *>(gs + place(row_tile(u)));
                const f16x4 lo = *reinterpret_cast<const f16x4 *>(gs + g_plane + place(row_tile(u)));
                poly[u] = acc * (c3 * (kScaleB / (kScaleA * kScaleA))) + joined(hi, lo) * (b * (kScaleB / kScaleA));
            });
        }
        __syncthreads();
        if (j < PT) {
#pragma unroll
            for (int u = 0; u < kT; ++u)
                if (wanted(u)) put(u, poly[u]);
        }
        __syncthreads();

        // X <- a X + B X, in the owner's registers
        if (wave < qt)
            row_tiles<PT>(gs + n * kSG + 8 * g, g_plane, kSG, kKP, xh, xl, [](int i) { return i; },
                          [&](int i, const f32x4 &acc) {
                              const int h = 4 * (i & 1);
                              const f16x4 hi = {xh[i >> 1][h], xh[i >> 1][h + 1], xh[i >> 1][h + 2], xh[i >> 1][h + 3]};
                              const f16x4 lo = {xl[i >> 1][h], xl[i >> 1][h + 1], xl[i >> 1][h + 2], xl[i >> 1][h + 3]};
                              x[i] = joined(hi, lo) * (a / kScaleX) + acc * (1.f / (kScaleB * kScaleX));
                          });
        // (the rows in LDS were last read before two barriers; B is next written after two more)
    }

    // to the caller, the weights in flight together
    const int step_r = tall ? 1 : io.ld, step_c = tall ? io.ld : 1;
    const int64_t from = base + (int64_t)min(own, q - 1) * step_c;
    f32x4 w[PT];
    if (io.w != nullptr) {
#pragma unroll
        for (int i = 0; i < PT; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) w[i][t] = io.w[from + (int64_t)min(16 * i + 4 * g + t, p - 1) * step_r];
#pragma unroll
        for (int i = 0; i < PT; ++i) x[i] = io.keep * w[i] - io.rate * x[i];
    }
    if (own < q) {
#pragma unroll
        for (int i = 0; i < PT; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (16 * i + 4 * g + t < p) io.out[from + (int64_t)(16 * i + 4 * g + t) * step_r] = x[i][t];
    }
}

template <int PT>
void launch_small(const OrthoIo &io, const Steps &steps, int count, hipStream_t stream) {
    const int p = std::min(io.rows, io.cols), q = std::max(io.rows, io.cols);
    if constexpr (PT <= 4)
        if (q <= 64) {
            hipLaunchKernelGGL((ortho_small_kernel<PT, 4>), dim3(count), dim3(256), (size_t)small_lds(p, q), stream, io, steps);
            return;
        }
    hipLaunchKernelGGL((ortho_small_kernel<PT, 8>), dim3(count), dim3(512), (size_t)small_lds(p, q), stream, io, steps);
}

int64_t aligned(int64_t n) { return (n + 255) / 256 * 256; }

template <int PT>
hipError_t small_attribute() {
    const int most = (int)small_lds(16 * PT, kSmall);
    if constexpr (PT <= 4) {
        const hipError_t e = hipFuncSetAttribute((const void *)ortho_small_kernel<PT, 4>,
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e != hipSuccess) return e;
    }
    return hipFuncSetAttribute((const void *)ortho_small_kernel<PT, 8>, hipFuncAttributeMaxDynamicSharedMemorySize, most);
}

}  // namespace

hipError_t set_ortho_attributes() {
    for (auto set : {small_attribute<1>, small_attribute<2>, small_attribute<3>, small_attribute<4>, small_attribute<5>,
                     small_attribute<6>, small_attribute<7>, small_attribute<8>}) {
        const hipError_t e = set();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int64_t ortho_bytes(int count, int rows, int cols) {
    if (std::max(rows, cols) <= kSmall) return 256;
    const OrthoShape sh = ortho_shape(rows, cols);
    return aligned(8 * (int64_t)count * norm_shares(rows, cols)) + 4 * aligned(4 * count * sh.x_plane()) +
           2 * aligned(4 * count * sh.a_plane());
}

hipError_t launch_ortho(const float *grad, const float *momentum, const float *w, float *momentum_out, float *out, int count,
                        int rows, int cols, int ld, float mu, bool nesterov, float keep, float rate, float eps,
                        const float *coefficients, int steps, char *ws, hipStream_t stream) {
    const OrthoShape sh = ortho_shape(rows, cols);
    OrthoIo io{grad, momentum, w, momentum_out, out, rows, cols, ld, mu, nesterov, keep, rate, eps};
    if (std::max(rows, cols) <= kSmall) {
        Steps all;
        all.count = steps;
        for (int k = 0; k < steps; ++k)
            for (int q = 0; q < 3; ++q) all.f[k][q] = coefficients[3 * k + q];
        void (*const by_tiles[])(const OrthoIo &, const Steps &, int, hipStream_t) = {
            launch_small<1>, launch_small<2>, launch_small<3>, launch_small<4>,
            launch_small<5>, launch_small<6>, launch_small<7>, launch_small<8>};
        by_tiles[(sh.p - 1) / 16](io, all, count, stream);
        return hipGetLastError();
    }
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
