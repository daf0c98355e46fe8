// crf_ortho.hip -- a matrix's nearest orthogonal one by Newton-Schulz products,
// and the update of weights by their orthogonalised momentum.
//
// With U the matrix (p rows, q >= p columns; a taller one is taken transposed),
//     X = U / (|U|_F + eps), and for each of the steps' (a, b, c):
//     A = X X^T,   B = a I + b A + c A A,   X <- B X,
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
// let the entries grow to, and no more.  Float32 itself is for matrices of up to
// 16 rows, which are bound by latency.
//
// Three ways, by size (five steps): thin matrices whole in registers (one of 16 x
// 1,000 in 26 us), small ones in a workgroup's LDS and registers (138 of 100 x 101
// in 46 us, 300 of 32 x 500 in 78), others a launch a product, tile by tile (one of
// 500 x 501 in 92 us, of 2,048 x 2,048 in 707).
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
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 64;   // sides are padded to multiples of this, or of twice it

// What X, A and B are held times: entries of at most 8, 32 and 64 fit float16.
constexpr float kScaleX = 4096.f, kScaleA = 2048.f, kScaleB = 1024.f;

// A stored matrix of rows of K entries lies in blocks of 32 rows x 16 entries,
// each an operand's fragment for the 64 lanes of a wavefront: a load or store of
// one is 1 KB on end.  A row of blocks has one to spare: workgroups read blocks of
// many of them at one place of K at a time, and a power of two between those
// would put them all on a few of the caches' and the memory's channels.
__host__ __device__ constexpr int64_t row_blocks(int K) { return K / 16 + 1; }

// Matrices of more rows and columns than this are padded to whole tiles of 128 x 128.
constexpr int kWide = 512;
// One matrix's arrays, each two planes (hi, then lo) of float16.
struct OrthoShape {
    int p, q;          // sides, p <= q
    int pp, qq;        // padded to whole tiles
    __host__ __device__ int64_t x_plane() const { return (int64_t)pp / 32 * row_blocks(qq) * 512; }
    __host__ __device__ int64_t xt_plane() const { return (int64_t)qq / 32 * row_blocks(pp) * 512; }
    __host__ __device__ int64_t a_plane() const { return (int64_t)pp / 32 * row_blocks(pp) * 512; }
};
__host__ __device__ inline OrthoShape ortho_shape(int rows, int cols) {
    OrthoShape s;
    s.p = rows < cols ? rows : cols;
    s.q = rows < cols ? cols : rows;
    const int pad = s.p > kWide ? 2 * kTile : kTile;
    s.pp = (s.p + pad - 1) / pad * pad;
    s.qq = (s.q + pad - 1) / pad * pad;
    return s;
}
// Shares of a matrix's norm: of kShareRows x 256 entries, or at most kMostShares.
constexpr int kShareRows = 4, kMostShares = 1024;
inline int norm_shares(int rows, int cols) {
    const int64_t size = (int64_t)rows * cols;
    return (int)std::min<int64_t>((size + 256 * kShareRows - 1) / (256 * kShareRows), kMostShares);
}

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
// (squares of float32 values neither overflow there nor vanish).  A workgroup
// takes every gridDim.x-th run of kShareRows x 256 entries.
__device__ __forceinline__ double sum_of_threads(double s, double *part) {
    part[threadIdx.x] = s;
    __syncthreads();
    for (int half = 128; half > 0; half /= 2) {
        if (threadIdx.x < half) part[threadIdx.x] += part[threadIdx.x + half];
        __syncthreads();
    }
    return part[0];
}
__global__ __launch_bounds__(256) void ortho_norm_kernel(OrthoIo io, double *__restrict__ shares) {
    __shared__ double part[256];
    const int64_t base = (int64_t)blockIdx.y * io.rows * io.ld;
    const int count = io.rows * io.cols;   // (at most 2^26)
    double s = 0.0;
    for (int first = blockIdx.x * 256 * kShareRows; first < count; first += gridDim.x * 256 * kShareRows) {
        int64_t at[kShareRows];
        float u[kShareRows], m[kShareRows];
#pragma unroll
        for (int e = 0; e < kShareRows; ++e) {
            const int k = min(first + 256 * e + (int)threadIdx.x, count - 1), row = k / io.cols;
            at[e] = base + (int64_t)row * io.ld + (k - row * io.cols);
            u[e] = io.grad[at[e]];
            if (io.momentum != nullptr) m[e] = io.momentum[at[e]];
        }
#pragma unroll
        for (int e = 0; e < kShareRows; ++e)
            if (first + 256 * e + (int)threadIdx.x < count) {
                if (io.momentum != nullptr) {
                    m[e] = fmaf(io.mu, m[e], u[e]);
                    io.momentum_out[at[e]] = m[e];
                    u[e] = updated(io, u[e], m[e]);
                }
                s += (double)u[e] * (double)u[e];
            }
    }
    s = sum_of_threads(s, part);
    if (threadIdx.x == 0) shares[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
}

__device__ __forceinline__ void split(const f32x4 &v, f16x4 &hi, f16x4 &lo) {
    hi = __builtin_convertvector(v, f16x4);
    lo = __builtin_convertvector(v - __builtin_convertvector(hi, f32x4), f16x4);
}
__device__ __forceinline__ void split(const float (&v)[8], f16x8 &hi, f16x8 &lo) {
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
        f16x4 a, b;
        split(f32x4{v[h], v[h + 1], v[h + 2], v[h + 3]}, a, b);
#pragma unroll
        for (int t = 0; t < 4; ++t) hi[h + t] = a[t], lo[h + t] = b[t];
    }
}
__device__ __forceinline__ f32x4 joined(const f16x4 &hi, const f16x4 &lo) {
    return __builtin_convertvector(hi, f32x4) + __builtin_convertvector(lo, f32x4);
}

// Where entries 8 c .. 8 c + 7 of row r (one lane's of a fragment) start.
__device__ __forceinline__ int64_t piece(int r, int c, int K) {
    return ((r >> 5) * row_blocks(K) + (c >> 1)) * 512 + ((r & 31) + 32 * (c & 1)) * 8;
}

// X = U / (|U|_F + eps) in parts, and its transpose; zeros past the matrix.
__global__ __launch_bounds__(256) void ortho_load_kernel(OrthoIo io, const double *__restrict__ shares, int n_shares,
                                                         _Float16 *__restrict__ x, _Float16 *__restrict__ xt) {
    __shared__ float tile[kTile][kTile + 1];
    __shared__ double part[256];
    const OrthoShape sh = ortho_shape(io.rows, io.cols);
    const bool tall = io.rows > io.cols;
    const int i0 = blockIdx.y * kTile, j0 = blockIdx.x * kTile;   // of X
    const int64_t base = (int64_t)blockIdx.z * io.rows * io.ld;
    float u[16], m[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {   // along the caller's rows, from their place 4 e + t / 64 on
        const int row = (tall ? j0 : i0) + 4 * e + ((int)threadIdx.x >> 6), col = (tall ? i0 : j0) + ((int)threadIdx.x & 63);
        const int64_t at = base + (int64_t)min(row, io.rows - 1) * io.ld + min(col, io.cols - 1);
        u[e] = io.grad[at];
        if (io.momentum != nullptr) m[e] = io.momentum_out[at];
    }
    double s = 0.0;
    for (int k = threadIdx.x; k < n_shares; k += 256) s += shares[(int64_t)blockIdx.z * n_shares + k];
    s = sum_of_threads(s, part);
    // (a sum that is not finite makes the whole matrix NaN)
    const double inv = (double)kScaleX / (sqrt(s) + (double)io.eps) + 0.0 * s;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int r = 4 * e + ((int)threadIdx.x >> 6), c = (int)threadIdx.x & 63;
        const bool there = (tall ? j0 : i0) + r < io.rows && (tall ? i0 : j0) + c < io.cols;
        const float v = io.momentum != nullptr ? updated(io, u[e], m[e]) : u[e];
        tile[tall ? c : r][tall ? r : c] = there ? (float)((double)v * inv) : 0.f;
    }
    __syncthreads();
    x += blockIdx.z * 2 * sh.x_plane();
    xt += blockIdx.z * 2 * sh.xt_plane();
    for (int e = threadIdx.x; e < kTile * kTile / 8; e += 256) {
        const int r = e % kTile, c = e / kTile;
        f16x8 hi, lo;
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = tile[r][8 * c + q];
        split(v, hi, lo);
        const int64_t at = piece(i0 + r, j0 / 8 + c, sh.qq), to = piece(j0 + r, i0 / 8 + c, sh.pp);
        *reinterpret_cast<f16x8 *>(x + at) = hi;
        *reinterpret_cast<f16x8 *>(x + sh.x_plane() + at) = lo;
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = tile[8 * c + q][r];
        split(v, hi, lo);
        *reinterpret_cast<f16x8 *>(xt + to) = hi;
        *reinterpret_cast<f16x8 *>(xt + sh.xt_plane() + to) = lo;
    }
}

// One tile of a product of two matrices whose rows run along K:
//   kGram  A = X X^T;      kPoly  B = a I + b A + c A A;
//   kNext  X' = B X (from B and X^T), and its transpose;   kLast  the same, to the caller.
// A and B are symmetric: a tile on or above the diagonal is computed, and stored
// as its mirror image too.
enum Product { kGram, kPoly, kNext, kLast };
struct ProductArgs {
    const _Float16 *left, *right;   // operands
    const _Float16 *add;            // A for kPoly
    _Float16 *out, *out_t;          // the result and its transpose
    int k, stride, t_stride;        // K; the entries of their rows
    int across;                     // tiles of a row of tiles
    int64_t left_plane, right_plane, out_plane, out_t_plane;
    float a, b, c;                  // in the scale of the result
};

// Workgroup's tile (i, j).
template <int KIND>
__device__ __forceinline__ void tile_of(const ProductArgs &g, int &i, int &j) {
    const int t = blockIdx.x;
    if constexpr (KIND == kGram || KIND == kPoly) {   // t = j (j + 1) / 2 + i, i <= j
        j = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
        while ((j + 1) * (j + 2) / 2 <= t) ++j;
        while (j * (j + 1) / 2 > t) --j;
        i = t - j * (j + 1) / 2;
    } else {
        i = t / g.across;
        j = t - i * g.across;
    }
}

__device__ __forceinline__ f16x8 frag(const _Float16 *p) { return *reinterpret_cast<const f16x8 *>(p); }

// What a tile's end reads from memory: A's entries or the weights of its places, a
// thread of NT's share.  Small tiles ask for it before the products.
template <int KIND, int T, int NT>
struct Held {
    static constexpr int kPieces = (T * T / 8 + NT - 1) / NT, kEntries = T * T / NT;   // a thread's
    f16x8 hi[KIND == kPoly ? kPieces : 1], lo[KIND == kPoly ? kPieces : 1];
    float w[KIND == kLast ? kEntries : 1];
    // entry e of the tile at (i0, j0), along the caller's rows; false: past the matrix
    static __device__ __forceinline__ bool entry(const OrthoIo &io, int i0, int j0, int e, int &at_tile, int64_t &at) {
        const bool tall = io.rows > io.cols;
        const int r = e / T, c = e % T, row = (tall ? j0 : i0) + r, col = (tall ? i0 : j0) + c;
        at_tile = tall ? c * (T + 1) + r : r * (T + 1) + c;
        at = (int64_t)blockIdx.z * io.rows * io.ld + (int64_t)row * io.ld + col;
        return row < io.rows && col < io.cols;
    }
    __device__ __forceinline__ void load(const ProductArgs &g, const OrthoIo &io, int i0, int j0) {
        if constexpr (KIND == kPoly) {
            const _Float16 *add = g.add + blockIdx.z * 2 * g.out_plane;
#pragma unroll
            for (int h = 0; h < kPieces; ++h) {
                const int e = min((int)threadIdx.x + h * NT, T * T / 8 - 1);
                const int64_t at = piece(i0 + e % T, j0 / 8 + e / T, g.stride);
                hi[h] = frag(add + at);
                lo[h] = frag(add + g.out_plane + at);
            }
        }
        if constexpr (KIND == kLast) {
            if (io.w == nullptr) return;
#pragma unroll
            for (int h = 0; h < kEntries; ++h) {
                int at_tile;
                int64_t at;
                w[h] = entry(io, i0, j0, threadIdx.x + h * NT, at_tile, at) ? io.w[at] : 0.f;
            }
        }
    }
};

// A tile's sums, in LDS at a row stride of T + 1, to where they belong: rows of
// the result, then (from LDS, so that both are whole lines) rows of its transpose.
template <int KIND, int T, int NT>
__device__ __forceinline__ void finish_tile(float *tile, const Held<KIND, T, NT> &held, const ProductArgs &g, const OrthoIo &io,
                                            int i0, int j0) {
    constexpr int kRow = T + 1;
    const int tid = threadIdx.x;
    if constexpr (KIND == kLast) {
#pragma unroll
        for (int h = 0; h < held.kEntries; ++h) {
            int from;
            int64_t to;
            if (held.entry(io, i0, j0, tid + h * NT, from, to)) {
                const float v = g.c * tile[from];
                io.out[to] = io.w != nullptr ? fmaf(-io.rate, v, io.keep * held.w[h]) : v;
            }
        }
        return;
    }
    const bool mirror = KIND == kNext || i0 != j0;
    _Float16 *out = g.out + blockIdx.z * 2 * g.out_plane;
#pragma unroll
    for (int h = 0; h < held.kPieces; ++h) {
        const int e = tid + h * NT, r = e % T, c = e / T;
        if (T * T / 8 < NT && e >= T * T / 8) break;
        const int64_t at = piece(i0 + r, j0 / 8 + c, g.stride);
        float *in = tile + r * kRow + 8 * c, v[8];
        f16x8 hi, lo;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            v[q] = in[q] * g.c;
            if constexpr (KIND == kPoly) {
                v[q] = fmaf(g.b, (float)held.hi[h][q] + (float)held.lo[h][q], v[q]);
                if (i0 + r == j0 + 8 * c + q) v[q] += g.a;
                if (mirror) in[q] = v[q];
            }
        }
        split(v, hi, lo);
        *reinterpret_cast<f16x8 *>(out + at) = hi;
        *reinterpret_cast<f16x8 *>(out + g.out_plane + at) = lo;
    }
    if (!mirror) return;
    if constexpr (KIND == kPoly) __syncthreads();
    _Float16 *out_t = g.out_t + blockIdx.z * 2 * g.out_t_plane;
#pragma unroll
    for (int h = 0; h < held.kPieces; ++h) {
        const int e = tid + h * NT, r = e % T, c = e / T;
        if (T * T / 8 < NT && e >= T * T / 8) break;
        const int64_t at = piece(j0 + r, i0 / 8 + c, g.t_stride);
        float v[8];
        f16x8 hi, lo;
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = tile[(8 * c + q) * kRow + r] * (KIND == kPoly ? 1.f : g.c);
        split(v, hi, lo);
        *reinterpret_cast<f16x8 *>(out_t + at) = hi;
        *reinterpret_cast<f16x8 *>(out_t + g.out_t_plane + at) = lo;
    }
}

// MFMA v_mfma_f32_32x32x16_f16: lane l supplies row l % 32 of either operand at K
// offsets 8 (l / 32) .. + 7, and holds rows 8 (t / 4) + 4 (l / 32) + t % 4 of
// column l % 32.
__device__ __forceinline__ void put_sums(float *tile, int stride, const f32x16 &acc, int lane) {
#pragma unroll
    for (int t = 0; t < 16; ++t) tile[(8 * (t >> 2) + 4 * (lane >> 5) + (t & 3)) * stride + (lane & 31)] = acc[t];
}

// Few tiles: 32 x 32 a workgroup, K split over its eight wavefronts, whose
// fragments come straight from L2 (each is used once), all in flight together up
// to K = 512, and whose sums meet in LDS.  A product of 500 x 501 takes 4 to 6 us, of
// which 2.5 are the launch and a fifth of one the matrix instructions.
constexpr int kFewTile = 32, kFewWaves = 8, kFewThreads = 64 * kFewWaves;
constexpr int kFewAhead = 4;   // steps of K (of 16) a wavefront has in flight
template <int KIND>
__global__ __launch_bounds__(kFewThreads) void ortho_few_kernel(ProductArgs g, OrthoIo io) {
    __shared__ float sums[kFewWaves][kFewTile * (kFewTile + 1)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int i, j;
    tile_of<KIND>(g, i, j);
    const int steps = g.k / 16, part = (steps + kFewWaves - 1) / kFewWaves;
    const int first = wave * part, end = min(first + part, steps);
    const _Float16 *left = g.left + blockIdx.z * 2 * g.left_plane + i * row_blocks(g.k) * 512 + 8 * lane;
    const _Float16 *right = g.right + blockIdx.z * 2 * g.right_plane + j * row_blocks(g.k) * 512 + 8 * lane;
    Held<KIND, kFewTile, kFewThreads> held;
    held.load(g, io, kFewTile * i, kFewTile * j);
    f32x16 acc[3];
#pragma unroll
    for (int t = 0; t < 3; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
    for (int s0 = first; s0 < end; s0 += kFewAhead) {
        f16x8 f[kFewAhead][4];
#pragma unroll
        for (int s = 0; s < kFewAhead; ++s) {
            const int64_t at = 512 * (int64_t)min(s0 + s, end - 1);
            f[s][0] = frag(left + at);
            f[s][1] = frag(left + g.left_plane + at);
            f[s][2] = frag(right + at);
            f[s][3] = frag(right + g.right_plane + at);
        }
#pragma unroll
        for (int s = 0; s < kFewAhead; ++s)
            if (s0 + s < end) {
                acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[s][0], f[s][3], acc[0], 0, 0, 0);
                acc[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[s][1], f[s][2], acc[1], 0, 0, 0);
                acc[2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[s][0], f[s][2], acc[2], 0, 0, 0);
            }
    }
    put_sums(sums[wave], kFewTile + 1, (acc[0] + acc[1]) + acc[2], lane);
    __syncthreads();
    for (int e = threadIdx.x; e < kFewTile * (kFewTile + 1); e += kFewThreads) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) s += sums[w][e];
        sums[0][e] = s;
    }
    __syncthreads();
    finish_tile<KIND, kFewTile, kFewThreads>(sums[0], held, g, io, kFewTile * i, kFewTile * j);
}

// Many: 64 M x 64 M a workgroup, a wavefront M x M tiles of 32 x 32.  Operands go
// through LDS 32 of K at a time, block by block as they lie, and all that a step
// does is for a later one: it loads step s + 2 + 2 M from memory into registers,
// stores step s + 2 to LDS, reads step s + 1's fragments and multiplies step s's,
// with one barrier.  (Read, multiplied and stored one after the other, with loads
// ahead alone, the four wavefronts of a CU leave the matrix cores idle for 60% of
// the time.)  2,048 x 2,048: B X takes 55 us, 940 TFLOP/s of float16, the matrix
// cores 64% busy at the clock that the card keeps then; 11 us of it are the stores.
constexpr int kStepK = 32, kRing = 3;
constexpr int kMfma = 0x008, kLoad = 0x020, kLdsRead = 0x100, kLdsWrite = 0x200;   // kinds of instructions to the scheduler
template <int M>
constexpr int staged_bytes() { return std::max(kRing * 16 * M * 1024, 64 * M * (64 * M + 1) * 4); }
template <int KIND, int M>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, M == 2 ? 1 : 3))) void ortho_tile_kernel(ProductArgs g,
                                                                                                     OrthoIo io) {
    constexpr int T = 64 * M, D = 2 * M, kPlane = 4 * M * 512, kBuffer = 4 * kPlane;   // left hi, lo, right hi, lo
    extern __shared__ __align__(16) char smem[];
    _Float16 *stage = reinterpret_cast<_Float16 *>(smem);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int i, j;
    tile_of<KIND>(g, i, j);
    // wavefront w moves blocks w + 4 h of each matrix's 4 M: row block / 2, K block
    const int64_t across = row_blocks(g.k);
    const _Float16 *left = g.left + blockIdx.z * 2 * g.left_plane + 2 * M * i * across * 512 + 8 * lane;
    const _Float16 *right = g.right + blockIdx.z * 2 * g.right_plane + 2 * M * j * across * 512 + 8 * lane;
    f16x8 next[D][4][M];
    auto load = [&](int d, int step) {   // (past the last step: the last one's again, which goes nowhere)
        const int k0 = min(step * kStepK, g.k - kStepK);
#pragma unroll
        for (int h = 0; h < M; ++h) {
            const int b = wave + 4 * h;
            const int64_t at = ((b >> 1) * across + k0 / 16 + (b & 1)) * 512;
            next[d][0][h] = frag(left + at);
            next[d][1][h] = frag(left + g.left_plane + at);
            next[d][2][h] = frag(right + at);
            next[d][3][h] = frag(right + g.right_plane + at);
        }
    };
    auto store = [&](int d, int buffer) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int h = 0; h < M; ++h)
                *reinterpret_cast<f16x8 *>(stage + buffer * kBuffer + s * kPlane + (wave + 4 * h) * 512 + 8 * lane) = next[d][s][h];
    };
    const int wi = 32 * M * (wave >> 1), wj = 32 * M * (wave & 1);   // the wavefront's part of the tile
    f16x8 l[2][2][2][M], r[2][2][2][M];   // of two steps: K block, part, tile
    auto read = [&](int w, int buffer) {
        const _Float16 *from = stage + buffer * kBuffer + 8 * lane;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    l[w][k][s][m] = frag(from + s * kPlane + (2 * (wi / 32 + m) + k) * 512);
                    r[w][k][s][m] = frag(from + (2 + s) * kPlane + (2 * (wj / 32 + m) + k) * 512);
                }
    };
    f32x16 acc[M][M];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int n = 0; n < M; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[m][n][e] = 0.f;
#pragma unroll
    for (int d = 0; d < D; ++d) load(d, d);
#pragma unroll
    for (int d = 0; d < 2; ++d) {
        store(d, d);
        load(d, d + D);
    }
    __syncthreads();
    read(0, 0);
    int ahead = 1, free = 2;   // buffers of steps s + 1 and s + 2
    for (int s0 = 0; s0 < g.k / kStepK; s0 += D)   // (K is a multiple of D steps, 64 M: see launch_product)
#pragma unroll
        for (int d = 0; d < D; ++d) {
            read((d + 1) & 1, ahead);
            store((d + 2) % D, free);
            load((d + 2) % D, s0 + d + 2 + D);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int s = 0; s < 3; ++s)   // hi lo, lo hi, hi hi
#pragma unroll
                    for (int m = 0; m < M; ++m)
#pragma unroll
                        for (int n = 0; n < M; ++n)
                            acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[d & 1][k][s == 1][m], r[d & 1][k][s == 0][n],
                                                                               acc[m][n], 0, 0, 0);
            // a wavefront issues in order: the others go between the products, or
            // the products wait for them
#pragma unroll
            for (int q = 0; q < (M == 2 ? 8 : 2); ++q) {
                __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kLdsRead, M == 2 ? 2 : 4, 0);
            }
#pragma unroll
            for (int q = 0; q < 4 * M; ++q) {
                __builtin_amdgcn_sched_group_barrier(kMfma, M, 0);
                __builtin_amdgcn_sched_group_barrier(kLdsWrite, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kLoad, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            __syncthreads();
            __builtin_amdgcn_sched_barrier(0);
            const int was = kRing - ahead - free;
            ahead = free;
            free = was;
        }
    __syncthreads();   // (the reads of a step past the last have ended)
    float *tile = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int n = 0; n < M; ++n) put_sums(tile + (wi + 32 * m) * (T + 1) + wj + 32 * n, T + 1, acc[m][n], lane);
    __syncthreads();
    Held<KIND, T, 256> held;
    held.load(g, io, T * i, T * j);
    finish_tile<KIND, T, 256>(tile, held, g, io, T * i, T * j);
}

// The largest tile that divides K and of which there are kEnoughTiles (half the CUs), or the least:
// five steps of one matrix of 640 x 640 take 110 us in tiles of 32 (134 of 64), of
// 1,024 x 1,024 183 of 64 (215 of 32, 331 of 128), of 1,536 x 1,536 418 of 128 for
// two products and 64 for the symmetric two (431 of 64, 450 of 128), of 2,048 x
// 2,048 707 of 128 (814 of 64, 1,254 of 32), 16 of 512 x 512 353 of 128 (392 of 64,
// 443 of 32).
constexpr int kEnoughTiles = 128;
template <int KIND>
void launch_product(const ProductArgs &args, const OrthoIo &io, int rows, int cols, int count, hipStream_t stream) {
    auto tiles = [&](int T) {
        const int64_t down = rows / T, across = cols / T;
        return KIND == kGram || KIND == kPoly ? down * (down + 1) / 2 : down * across;
    };
    // (a tile of T takes K in rounds of T: X X^T runs along qq, which a result of
    // pp x pp says nothing of)
    auto fits = [&](int T) {
        return rows % T == 0 && cols % T == 0 && args.k % T == 0 && tiles(T) * count >= kEnoughTiles;
    };
    ProductArgs g = args;
    const int T = fits(128) ? 128 : fits(64) ? 64 : kFewTile;
    g.across = cols / T;
    const dim3 grid((uint32_t)tiles(T), 1, count);
    if (T == kFewTile)
        hipLaunchKernelGGL(ortho_few_kernel<KIND>, grid, dim3(kFewThreads), 0, stream, g, io);
    else if (T == 64)
        hipLaunchKernelGGL((ortho_tile_kernel<KIND, 1>), grid, dim3(256), staged_bytes<1>(), stream, g, io);
    else
        hipLaunchKernelGGL((ortho_tile_kernel<KIND, 2>), grid, dim3(256), staged_bytes<2>(), stream, g, io);
}

struct Steps {
    float f[CRF_MAX_STEPS][3];
    int count;
};

// Matrices of up to 16 x 2,048: a workgroup of W wavefronts each, a wavefront C of
// X's tiles of 16 columns, and float32's own matrix instruction (the parts of 22
// bits, and not its length, are what 16 rows' error comes from: 1.1e-6 against
// 0.7e-6 on 155 x 7).  Its result has, a lane l, rows 4 (l / 16) + t of column
// l % 16, t = 0 .. 3, and its operand t is a row of K for a lane l / 16: so a
// result's register t is operand t of a product that runs K in the order 0, 4, 8,
// 12 | 1, 5 .., as the right one, and as the left one it is the transpose.  Hence
// X^T B from X and B, X X^T from X^T, B X from the symmetric B and X, all without
// leaving the registers; only the wavefronts' sums of A meet in LDS, once a step.
// (Five steps of one 16 x 1,000: 26 us, as parts in LDS 39; of 300 of them 47, 80.)
constexpr int kThinRows = 16, kThinCols = 2048;
inline bool is_thin(int rows, int cols) { return std::min(rows, cols) <= kThinRows && std::max(rows, cols) <= kThinCols; }
// left^T right (+ acc)
__device__ __forceinline__ f32x4 times(const f32x4 &left, const f32x4 &right, f32x4 acc) {
#pragma unroll
    for (int t = 0; t < 4; ++t) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(left[t], right[t], acc, 0, 0, 0);
    return acc;
}
template <int W, int C>
__global__ __launch_bounds__(64 * W) void ortho_thin_kernel(OrthoIo io, Steps steps) {
    __shared__ f32x4 part[2][W][64];
    __shared__ double norm[W];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int n = lane & 15;
    const int g = lane >> 4;
    const bool tall = io.rows > io.cols;
    const int p = tall ? io.cols : io.rows, q = tall ? io.rows : io.cols;
    const int64_t step_r = tall ? 1 : io.ld, step_c = tall ? io.ld : 1;   // of X, in the caller's arrays
    int64_t row[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) row[t] = min(4 * g + t, p - 1) * step_r + (int64_t)blockIdx.x * io.rows * io.ld;
    auto tile = [&](int c) { return c * W + wave; };
    auto column = [&](int c) { return min(16 * tile(c) + n, q - 1) * step_c; };
    auto there = [&](int c, int t) { return 4 * g + t < p && 16 * tile(c) + n < q; };
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    // U, the new momentum and the norm
    f32x4 x[C], m[C];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            x[c][t] = io.grad[row[t] + column(c)];
            m[c][t] = io.momentum != nullptr ? io.momentum[row[t] + column(c)] : 0.f;
        }
    asm("" : "+v"(n));   // (places are worked out again, here and below: kept for all columns, they spill)
    double sum = 0.0;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (io.momentum != nullptr) {
                m[c][t] = fmaf(io.mu, m[c][t], x[c][t]);
                if (there(c, t)) io.momentum_out[row[t] + column(c)] = m[c][t];
                x[c][t] = updated(io, x[c][t], m[c][t]);
            }
            x[c][t] = there(c, t) ? x[c][t] : 0.f;
            sum += (double)x[c][t] * (double)x[c][t];
        }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
    if constexpr (W > 1) {
        if (lane == 0) norm[wave] = sum;
        __syncthreads();
        sum = norm[0];
#pragma unroll
        for (int w = 1; w < W; ++w) sum += norm[w];
    }
    // (a sum that is not finite makes the whole matrix NaN)
    const double inv = 1.0 / (sqrt(sum) + (double)io.eps) + 0.0 * sum;
    f32x4 one, gram[2] = {zero, zero};   // the wavefront's sum of A, in two chains
#pragma unroll
    for (int t = 0; t < 4; ++t) one[t] = 4 * g + t == n ? 1.f : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int t = 0; t < 4; ++t) x[c][t] = (float)((double)x[c][t] * inv);
        const f32x4 xt = times(x[c], one, zero);   // (exact)
        gram[c & 1] = times(xt, xt, gram[c & 1]);
    }

    asm("" : "+v"(n));
    for (int k = 0; k < steps.count; ++k) {
        f32x4 a = gram[0] + gram[1];
        if constexpr (W > 1) {
            part[k & 1][wave][lane] = a;   // (the readers of step k - 2 are past the last step's barrier)
            __syncthreads();
            a = part[k & 1][0][lane];
#pragma unroll
            for (int w = 1; w < W; ++w) a += part[k & 1][w][lane];
        }
        const f32x4 square = times(a, a, zero);
        f32x4 b;
#pragma unroll
        for (int t = 0; t < 4; ++t) b[t] = fmaf(steps.f[k][2], square[t], fmaf(steps.f[k][1], a[t], steps.f[k][0] * one[t]));
        gram[0] = gram[1] = zero;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const f32x4 xt = times(x[c], b, zero);
            x[c] = times(b, x[c], zero);
            gram[c & 1] = times(xt, xt, gram[c & 1]);   // (after the last step nobody asks)
        }
    }

    asm("" : "+v"(n));
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int t = 0; t < 4; ++t) m[c][t] = io.w != nullptr ? io.w[row[t] + column(c)] : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (there(c, t)) io.out[row[t] + column(c)] = io.w != nullptr ? fmaf(-io.rate, x[c][t], io.keep * m[c][t]) : x[c][t];
}

template <int W, int C>
void launch_thin_c(const OrthoIo &io, const Steps &steps, int count, hipStream_t stream) {
    hipLaunchKernelGGL((ortho_thin_kernel<W, C>), dim3(count), dim3(64 * W), 0, stream, io, steps);
}
void launch_thin(const OrthoIo &io, const Steps &steps, int count, hipStream_t stream) {
    const int q = std::max(io.rows, io.cols);
    (q <= 16     ? launch_thin_c<1, 1>
     : q <= 64   ? launch_thin_c<4, 1>
     : q <= 128  ? launch_thin_c<8, 1>
     : q <= 256  ? launch_thin_c<8, 2>
     : q <= 384  ? launch_thin_c<8, 3>
     : q <= 512  ? launch_thin_c<8, 4>
     : q <= 768  ? launch_thin_c<8, 6>
     : q <= 1024 ? launch_thin_c<8, 8>
     : q <= 1536 ? launch_thin_c<8, 12>
                 : launch_thin_c<8, 16>)(io, steps, count, stream);
}

// More rows, whose parts fit LDS twice over: a workgroup of W wavefronts each, which
// never leaves its CU.  Wavefront w owns C of X's tiles of 16 columns, w, w + W ..,
// in registers.  Their parts are wanted twice over: in LDS, as rows of X, for the
// Gram matrix, and in the owner's registers as the right operand of B X -- a
// product's result has, a lane, four consecutive rows of one column, and two
// tiles of it are just a right operand's fragment whose K runs 0-3, 16-19 | 4-7,
// 20-23 | ...; the Gram matrix and B are stored with their columns in that order,
// so that no product minds.  A and B are symmetric: of the tiles (i, j) and (j, i)
// one is computed, column j taking rows j, j + 1 .. j + PT / 2 (cyclically), which
// shares the work evenly.  Bound by a step's three chains (products, LDS, barrier):
// 6.6 us a step of 100 x 101 whether there is one matrix or 138, the matrix cores
// 23% busy; 300 of 100 x 150 take 116 us, a launch a product 351, 300 of 32 x 500
// 78 and 221.
constexpr int kSmallRows = 128;
__host__ __device__ constexpr int small_stride(int tiles) { return (tiles + 1) / 2 * 32 + 8; }   // of a row of 16 `tiles`
inline int64_t small_lds(int p, int q) {
    const int pt = (p + 15) / 16, qt = (q + 15) / 16;
    return std::max<int64_t>(2 * 2 * 2 * 16 * pt * (int64_t)small_stride(qt), 4 * (int64_t)q * (p + 1));
}
// Column tiles of a wavefront of eight, for `pt` row tiles at most.
constexpr int small_most(int pt) { return pt <= 3 ? 4 : pt <= 7 ? 2 : 1; }
inline bool is_small(int rows, int cols) {
    const int p = std::min(rows, cols), q = std::max(rows, cols);
    return p <= kSmallRows && (q + 127) / 128 <= small_most((p + 15) / 16) && small_lds(p, q) <= 160 * 1024 - 256;
}

// U row tiles of a stored matrix (hi, and lo `plane` entries on) times a column
// tile in registers: tile u is at row tile row(u), and done(u, acc) takes its
// result.  ks: steps of K.  The next tile's fragments fly while this one's
// products run, in a chain for each of the three, and the last one's result is
// taken.
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
    f32x4 acc[2][3];
    auto sum = [&](int u) { return (acc[u & 1][0] + acc[u & 1][1]) + acc[u & 1][2]; };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (u + 1 < U) load(u + 1);
#pragma unroll
        for (int t = 0; t < 3; ++t) acc[u & 1][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s)
            if (s < ks) {
                acc[u & 1][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lh[u & 1][s], rl[s], acc[u & 1][0], 0, 0, 0);
                acc[u & 1][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ll[u & 1][s], rh[s], acc[u & 1][1], 0, 0, 0);
                acc[u & 1][2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lh[u & 1][s], rh[s], acc[u & 1][2], 0, 0, 0);
            }
        if (u > 0) done(u - 1, sum(u - 1));
        __builtin_amdgcn_sched_barrier(0);   // (no further loads ahead: their registers spill)
    }
    done(U - 1, sum(U - 1));
}

template <int PT, int W, int C>
__global__ __launch_bounds__(64 * W) void ortho_small_kernel(OrthoIo io, Steps steps) {
    constexpr int kKP = (PT + 1) / 2;          // steps of K over p
    constexpr int kKQ = C == 1 ? W / 2 : 4;    // of K over q at a time
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
    const int x_plane = 16 * PT * sx;   // (no less than a plane of A's: q >= p)
    constexpr int g_plane = 16 * PT * kSG;
    _Float16 *xs = reinterpret_cast<_Float16 *>(smem), *gs = xs + 2 * x_plane;
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
    // X's parts, tile (i, c): rows 16 i + 4 g .. + 3 of column 16 tile(c) + n
    f16x8 xh[C][kKP], xl[C][kKP];
    auto tile = [&](int c) { return c * W + wave; };
    auto set = [&](f16x8 (&hi8)[kKP], f16x8 (&lo8)[kKP], int i, const f16x4 &hi, const f16x4 &lo) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            hi8[i >> 1][4 * (i & 1) + t] = hi[t];
            lo8[i >> 1][4 * (i & 1) + t] = lo[t];
        }
    };
    auto get = [&](const f16x8 (&v)[kKP], int i) {
        const int h = 4 * (i & 1);
        return f16x4{v[i >> 1][h], v[i >> 1][h + 1], v[i >> 1][h + 2], v[i >> 1][h + 3]};
    };
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 2 * kKP; ++i) {
            f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int r = 16 * i + 4 * g + t, col = 16 * tile(c) + n, row = min(r, p - 1), at = min(col, q - 1);
                const float u = (float)((double)us[tall ? at * us_stride + row : row * us_stride + at] * inv);
                x[t] = r < p && col < q ? u : 0.f;
            }
            f16x4 hi, lo;
            split(kScaleX * x, hi, lo);
            set(xh[c], xl[c], i, hi, lo);
        }
    __syncthreads();
    // (what lies past the tiles in the last step of K is multiplied by zeros, so it has to be finite)
    for (int k = tid; k < 4 * x_plane / 8; k += kThreads) reinterpret_cast<u32x4 *>(xs)[k] = u32x4{0u, 0u, 0u, 0u};
    __syncthreads();
    // a tile's parts into the rows of X
    auto put_x = [&](_Float16 *to, int i, int c, const f16x4 &hi, const f16x4 &lo) {
        to += (16 * i + 4 * g) * sx + 16 * tile(c) + n;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            to[t * sx] = hi[t];
            to[x_plane + t * sx] = lo[t];
        }
    };
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (tile(c) < qt) {
#pragma unroll
            for (int i = 0; i < PT; ++i) put_x(xs, i, c, get(xh[c], i), get(xl[c], i));
        }
    __syncthreads();

    // X lies in xs; A goes to gs, B to xs, and the new X to gs: each is read by all
    // wavefronts before the barrier after which its place is written
#pragma unroll 1
    for (int step = 0; step < steps.count; ++step) {
        const float a = steps.f[step][0], b = steps.f[step][1], c3 = steps.f[step][2];
        // (a step's LDS addresses are taken from these anew: kept over the loop,
        // some hundred of them, they would take the registers that X lies in)
        asm("" : "+v"(n), "+v"(g));

        // Symmetric products: column tile j, row tiles j + u (cyclically)
        const int j = wave;
        auto row_tile = [&](int u) { return j + u < PT ? j + u : j + u - PT; };
        auto wanted = [&](int u) { return PT % 2 != 0 || u < PT / 2 || j < PT / 2; };
        // where tile (i, j)'s lane puts its four rows: row 16 j + n of the stored
        // matrix, columns 16 i + 4 g .. + 3 in their order, and the mirror image
        auto place = [&](int i) { return (16 * j + n) * kSG + 32 * (i >> 1) + 8 * g + 4 * (i & 1); };
        auto put = [&](_Float16 *to, int u, const f32x4 &v) {
            const int i = row_tile(u);
            f16x4 hi, lo;
            split(v, hi, lo);
            *reinterpret_cast<f16x4 *>(to + place(i)) = hi;
            *reinterpret_cast<f16x4 *>(to + g_plane + place(i)) = lo;
            if (u > 0) {
                const int at = (16 * i + 4 * g) * kSG + 32 * (j >> 1) + 8 * (n >> 2) + 4 * (j & 1) + (n & 3);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    to[at + t * kSG] = hi[t];
                    to[g_plane + at + t * kSG] = lo[t];
                }
            }
        };

        // A = X X^T
        if (j < PT) {
            f16x8 rh[kKQ], rl[kKQ];
            auto columns = [&](int s0) {
#pragma unroll
                for (int s = 0; s < kKQ; ++s)
                    if (s0 + s < kq) {
                        const _Float16 *from = xs + (16 * j + n) * sx + 32 * (s0 + s) + 8 * g;
                        rh[s] = frag(from);
                        rl[s] = frag(from + x_plane);
                        if (2 * (s0 + s) + 1 == qt && g >= 2) rh[s] = rl[s] = f16x8{0, 0, 0, 0, 0, 0, 0, 0};
                    }
            };
            auto done = [&](int u, const f32x4 &acc) {
                if (wanted(u)) put(gs, u, acc * (kScaleA / (kScaleX * kScaleX)));
            };
            if constexpr (C == 1) {
                columns(0);
                row_tiles<kT>(xs + n * sx + 8 * g, x_plane, sx, kq, rh, rl, row_tile, done);
            } else {   // all row tiles' sums together, kKQ steps of K at a time
                f32x4 acc[kT][3];
#pragma unroll
                for (int u = 0; u < kT; ++u)
#pragma unroll
                    for (int t = 0; t < 3; ++t) acc[u][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int s0 = 0; s0 < kq; s0 += kKQ) {
                    columns(s0);
#pragma unroll
                    for (int u = 0; u < kT; ++u)
#pragma unroll
                        for (int s = 0; s < kKQ; ++s)
                            if (s0 + s < kq) {
                                const _Float16 *at = xs + (16 * row_tile(u) + n) * sx + 32 * (s0 + s) + 8 * g;
                                const f16x8 lh = frag(at), ll = frag(at + x_plane);
                                acc[u][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lh, rl[s], acc[u][0], 0, 0, 0);
                                acc[u][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ll, rh[s], acc[u][1], 0, 0, 0);
                                acc[u][2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lh, rh[s], acc[u][2], 0, 0, 0);
                            }
                }
#pragma unroll
                for (int u = 0; u < kT; ++u) done(u, (acc[u][0] + acc[u][1]) + acc[u][2]);
            }
        }
        __syncthreads();

        // B = a I + b A + c A A
        if (j < PT) {
            f16x8 rh[kKP], rl[kKP];
#pragma unroll
            for (int s = 0; s < kKP; ++s) {
                const _Float16 *from = gs + (16 * j + n) * kSG + 32 * s + 8 * g;
                rh[s] = frag(from);
                rl[s] = frag(from + g_plane);
            }
            if constexpr (PT % 2 != 0) {
#pragma unroll
                for (int t = 4; t < 8; ++t) rh[kKP - 1][t] = rl[kKP - 1][t] = (_Float16)0.f;
            }
            row_tiles<kT>(gs + n * kSG + 8 * g, g_plane, kSG, kKP, rh, rl, row_tile, [&](int u, const f32x4 &acc) {
                const f16x4 hi = *reinterpret_cast<const f16x4 *>(gs + place(row_tile(u)));
                const f16x4 lo = *reinterpret_cast<const f16x4 *>(gs + g_plane + place(row_tile(u)));
                f32x4 v = acc * (c3 * (kScaleB / (kScaleA * kScaleA))) + joined(hi, lo) * (b * (kScaleB / kScaleA));
                if (u == 0) {
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (4 * g + t == n) v[t] += a * kScaleB;
                }
                if (wanted(u)) put(xs, u, v);
            });
        }
        __syncthreads();

        // X <- B X, in the owner's registers, a column tile at a time
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (tile(c) < qt) {
                f16x8 nh[kKP], nl[kKP];
                if constexpr (PT % 2 != 0) set(nh, nl, PT, f16x4{0, 0, 0, 0}, f16x4{0, 0, 0, 0});
                row_tiles<PT>(xs + n * kSG + 8 * g, g_plane, kSG, kKP, xh[c], xl[c], [](int i) { return i; },
                              [&](int i, const f32x4 &acc) {
                                  f16x4 hi, lo;
                                  split(acc * (1.f / kScaleB), hi, lo);
                                  set(nh, nl, i, hi, lo);
                                  put_x(gs, i, c, hi, lo);
                              });
#pragma unroll
                for (int s = 0; s < kKP; ++s) xh[c][s] = nh[s], xl[c][s] = nl[s];
            }
        __syncthreads();
        _Float16 *was = xs;
        xs = gs;
        gs = was;
    }

    // to the caller, a column tile's weights in flight together
    const int step_r = tall ? 1 : io.ld, step_c = tall ? io.ld : 1;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int own = 16 * tile(c) + n;
        const int64_t from = base + (int64_t)min(own, q - 1) * step_c;
        f32x4 x[PT], w[PT];
#pragma unroll
        for (int i = 0; i < PT; ++i) x[i] = joined(get(xh[c], i), get(xl[c], i)) * (1.f / kScaleX);
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
}

template <int PT, int W, int C>
void launch_small_c(const OrthoIo &io, const Steps &steps, int count, hipStream_t stream) {
    hipLaunchKernelGGL((ortho_small_kernel<PT, W, C>), dim3(count), dim3(64 * W),
                       (size_t)small_lds(std::min(io.rows, io.cols), std::max(io.rows, io.cols)), stream, io, steps);
}
template <int PT>
void launch_small(const OrthoIo &io, const Steps &steps, int count, hipStream_t stream) {
    const int q = std::max(io.rows, io.cols);
    if constexpr (PT <= 4)
        if (q <= 64) return launch_small_c<PT, 4, 1>(io, steps, count, stream);
    if (q <= 128) return launch_small_c<PT, 8, 1>(io, steps, count, stream);
    if constexpr (small_most(PT) >= 2)
        if (q <= 256) return launch_small_c<PT, 8, 2>(io, steps, count, stream);
    if constexpr (small_most(PT) >= 4) launch_small_c<PT, 8, 4>(io, steps, count, stream);
}

int64_t aligned(int64_t n) { return (n + 255) / 256 * 256; }

template <int KIND>
hipError_t tile_attribute() {
    return hipFuncSetAttribute((const void *)ortho_tile_kernel<KIND, 2>, hipFuncAttributeMaxDynamicSharedMemorySize,
                               staged_bytes<2>());
}
template <int PT>
hipError_t small_attribute() {
    auto set = [](const void *f) {
        return hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024 - 256);
    };
    hipError_t e = set((const void *)ortho_small_kernel<PT, 8, 1>);
    if constexpr (PT <= 4)
        if (e == hipSuccess) e = set((const void *)ortho_small_kernel<PT, 4, 1>);
    if constexpr (small_most(PT) >= 2)
        if (e == hipSuccess) e = set((const void *)ortho_small_kernel<PT, 8, 2>);
    if constexpr (small_most(PT) >= 4)
        if (e == hipSuccess) e = set((const void *)ortho_small_kernel<PT, 8, 4>);
    return e;
}

}  // namespace

hipError_t set_ortho_attributes() {
    for (auto set : {small_attribute<2>, small_attribute<3>, small_attribute<4>, small_attribute<5>, small_attribute<6>,
                     small_attribute<7>, small_attribute<8>, tile_attribute<kGram>, tile_attribute<kPoly>, tile_attribute<kNext>,
                     tile_attribute<kLast>}) {
        const hipError_t e = set();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int64_t ortho_bytes(int count, int rows, int cols) {
    if (is_thin(rows, cols) || is_small(rows, cols)) return 256;
    const OrthoShape sh = ortho_shape(rows, cols);
    return aligned(8 * (int64_t)count * norm_shares(rows, cols)) + 2 * aligned(4 * count * sh.x_plane()) +
           2 * aligned(4 * count * sh.xt_plane()) + 2 * aligned(4 * count * sh.a_plane());
}

hipError_t launch_ortho(const float *grad, const float *momentum, const float *w, float *momentum_out, float *out, int count,
                        int rows, int cols, int ld, float mu, bool nesterov, float keep, float rate, float eps,
                        const float *coefficients, int steps, char *ws, hipStream_t stream) {
    const OrthoShape sh = ortho_shape(rows, cols);
    OrthoIo io{grad, momentum, w, momentum_out, out, rows, cols, ld, mu, nesterov, keep, rate, eps};
    if (is_thin(rows, cols) || is_small(rows, cols)) {
        Steps all;
        all.count = steps;
        for (int k = 0; k < steps; ++k)
            for (int q = 0; q < 3; ++q) all.f[k][q] = coefficients[3 * k + q];
        void (*const by_tiles[])(const OrthoIo &, const Steps &, int, hipStream_t) = {
            launch_thin,     launch_small<2>, launch_small<3>, launch_small<4>,
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
    for (int k = 0; k < 2; ++k) x[k] = take(sh.x_plane()), xt[k] = take(sh.xt_plane());
    a = take(sh.a_plane());
    b = take(sh.a_plane());
    const int n_shares = norm_shares(rows, cols);
    hipLaunchKernelGGL(ortho_norm_kernel, dim3(n_shares, count), dim3(256), 0, stream, io, shares);
    hipLaunchKernelGGL(ortho_load_kernel, dim3(sh.qq / kTile, sh.pp / kTile, count), dim3(256), 0, stream, io, shares,
                       n_shares, x[0], xt[0]);
    for (int s = 0; s < steps; ++s) {
        const float *co = coefficients + 3 * s;
        const int now = s & 1;
        const ProductArgs gram{x[now], x[now], nullptr, a, a, sh.qq, sh.pp, sh.pp, 0, sh.x_plane(), sh.x_plane(), sh.a_plane(),
                               sh.a_plane(), 0.f, 0.f, kScaleA / (kScaleX * kScaleX)};
        const ProductArgs poly{a, a, a, b, b, sh.pp, sh.pp, sh.pp, 0, sh.a_plane(), sh.a_plane(), sh.a_plane(),
                               sh.a_plane(), co[0] * kScaleB, co[1] * (kScaleB / kScaleA), co[2] * (kScaleB / (kScaleA * kScaleA))};
        ProductArgs next{b, xt[now], nullptr, x[now ^ 1], xt[now ^ 1], sh.pp, sh.qq, sh.pp, 0, sh.a_plane(), sh.xt_plane(),
                         sh.x_plane(), sh.xt_plane(), 0.f, 0.f, 1.f / kScaleB};
        launch_product<kGram>(gram, io, sh.pp, sh.pp, count, stream);
        launch_product<kPoly>(poly, io, sh.pp, sh.pp, count, stream);
        if (s + 1 == steps) {
            next.c /= kScaleX;
            launch_product<kLast>(next, io, sh.pp, sh.qq, count, stream);
        } else {
            launch_product<kNext>(next, io, sh.pp, sh.qq, count, stream);
        }
    }
    return hipGetLastError();
}

}  // namespace crf
