// crf_biaffine_bwd.hip -- the backward pass of the biaffine scorer.
//
// The scorer (crf_biaffine.hip) forms s(i,j,l) = [r^l_i ; 1]^T W_l r^r_j.  With
// G_l(i,j) = dL/ds(i,j,l) on the spans i < j <= n of a sentence,
//     U_l = G_l R^r,   X_l = G_l^T [R^l ; 1]           (posts x d, posts x (d+1))
//     dR^l = sum_l U_l W_l^T (its first d columns),  dR^r = sum_l X_l W_l,
//     dW_l = [R^l ; 1]^T U_l, summed over the batch's posts.
// The products with G run inside blocks of 64 fence posts (KernelPlan::posts:
// short sentences packed whole, longer ones cut, a block then meeting every
// block of its sentence on its side of the diagonal), so that what they cost
// is small beside the three dense products.  Blocks of whole sentences multiply
// by W first, dR^l = G (R^r W^T) and dR^r = G^T ([R^l ; 1] W), which keeps that
// product in registers; blocks of longer ones by G first (U and X above), so
// that the dense product is not repeated for each partner.
//
// What bounds it: the matrix cores, as far as staging lets them.  5,000
// sentences (130,000 posts) at d = 500 need 2e11 operations, 160 us at the
// 1.24e15 a second of a large library product, and 0.5 GB, 103 us.  A call
// takes 446 us, from 8-bit rows 444.  Kernel by kernel, profiled in ten calls
// from cold: rows 207 (whole sentences) and 29 (long ones), dW 252 and the sum
// of its shares 11, W's fragments 5; all figures below are of such profiles.
//
// Roundings.  R and W are bf16, products and sums fp32.  G, which is fp32, goes
// in as bf16 hi + lo parts (at most 2^-16 of it is lost), and so does the inner
// product, R W or G R, into the outer one.  dW comes out in fp32, dR^l and dR^r
// in bf16, their one rounding of that size.  (With one bf16 part of the inner
// product of dR they were 2.4e-3 off, and 1.7e-3 is bf16's own.  The second part
// makes the small product with G half as long again, and the long sentences'
// dense one twice as long: 5,000 sentences at d = 500 rows 207 us either way and
// long ones 23 -> 29, 138 labels of 100 sentences at d = 100 63 -> 73 and 38 -> 43.)
//
// MFMA v_mfma_f32_16x16x32_bf16: lane l supplies A row l%16 and B column l%16
// at K offsets 8(l/16)..+7 and holds D rows 4(l/16)..+3 of column l%16.  An
// operand whose K runs over rows of LDS is read with ds_read_b64_tr_b16: of a
// group of 16 lanes, lane s reads four neighbours of row s/4 from column
// 4(s%4), and receives of the 4 x 16 block the four rows of column s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "crf_internal.h"
#include "crf_rows.h"

namespace crf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kBlk = kBiaRows;               // fence posts of a block
constexpr int kGS = kBlk + 4;                // row stride of the staged G

__device__ __forceinline__ bf16x8 frag(const uint16_t *p) {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(p));
}
// K offsets 0..3 and 4..7 of an operand from rows of LDS: p0 and p1 the
// addresses of this lane's part of the two 4 x 16 blocks.
__device__ __forceinline__ bf16x8 frag_rows(const uint16_t *p0, const uint16_t *p1) {
    typedef __attribute__((address_space(3))) s16x4 lds_t;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(p0));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(p1));
    const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
    return __builtin_bit_cast(bf16x8, make_uint4(x.x, x.y, y.x, y.y));
}
__device__ __forceinline__ f32x4 mfma(const bf16x8 &a, const bf16x8 &b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Two float32 as bf16 parts hi + lo.
__device__ __forceinline__ void parts(float a, float b, uint32_t &hi, uint32_t &lo) {
    hi = two_bf16(a, b);
    lo = two_bf16(a - __builtin_bit_cast(float, hi << 16), b - __builtin_bit_cast(float, hi & 0xFFFF0000u));
}

// Two fours of a lane as an operand's eight, as bf16 parts hi + lo.
__device__ __forceinline__ void two_parts(const f32x4 &x, const f32x4 &y, bf16x8 &hi, bf16x8 &lo) {
    uint4 h, l;
    parts(x[0], x[1], h.x, l.x);
    parts(x[2], x[3], h.y, l.y);
    parts(y[0], y[1], h.z, l.z);
    parts(y[2], y[3], h.w, l.w);
    hi = __builtin_bit_cast(bf16x8, h);
    lo = __builtin_bit_cast(bf16x8, l);
}

// Representations as the caller holds them: bf16 rows, or 8-bit codes and
// their scales (crf_rows.h).
struct Rows {
    const void *x;
    const uint8_t *scales;
    int last;   // the last row that 16 bytes of bf16 can be read from (see Staged)
};
// The plan's tables are constant while a kernel runs: scalar loads where the
// address is uniform.
template <typename T>
__device__ __forceinline__ T constant(const T *p) {
    return *(const __attribute__((address_space(4))) T *)p;
}

// Staging goes through registers: loads first, without a branch (addresses that
// hold nothing for a lane are moved to ones that exist, and what comes from
// there is left out when it is stored), so that all of them are in flight
// together until the products of the step before are done.  (A branch around
// each load made the compiler wait for it there: 5,000 sentences at d = 500,
// rows 418 us.)
//
// Columns k0 .. k0 + COLS of the rows of a block, to LDS with row stride
// `stride`: wavefront w of NW takes kRows rows from kRows w on, whose ids are
// then scalars, kAtOnce of them side by side, a lane eight entries of each.
template <int COLS, int NW, bool Q8>
struct Staged {
    static constexpr int kRows = kBlk / NW;
    static constexpr int kPieces = COLS / 8;                                  // of a row
    static constexpr int kAtOnce = kPieces <= 32 ? 64 / kPieces : 1;          // rows
    static constexpr int kEach = kRows / kAtOnce;
    uint4 v[kEach];   // (Q8: codes in x and y, the scale in z)
    int id[kRows];
    static __device__ __forceinline__ int row(int u) {   // within the wavefront's
        return kAtOnce * u + (kAtOnce > 1 ? (int)(threadIdx.x & 63) / kPieces : 0);
    }
    static __device__ __forceinline__ int col() {
        const int lane = threadIdx.x & 63;
        return 8 * (kAtOnce > 1 ? lane % kPieces : kPieces < 64 ? min(lane, kPieces - 1) : lane);
    }
    __device__ __forceinline__ int id_of(int u) const {
        int x = id[kAtOnce * u];
        if constexpr (kAtOnce > 1) {   // (masks: a choice would be one of addresses, and the ids in memory)
            const int q = (int)(threadIdx.x & 63) / kPieces;
#pragma unroll
            for (int t = 1; t < kAtOnce; ++t) {
                const int m = q == t ? -1 : 0;
                x = (x & ~m) | (id[kAtOnce * u + t] & m);
            }
        }
        return x;
    }
    // post: the block's record
    __device__ __forceinline__ void load(const Rows &r, const int32_t *post, int k0, int d) {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        int k = k0 + col();
#pragma unroll
        for (int u = 0; u < kRows; ++u) id[u] = constant(post + kRows * w + u);
        if constexpr (Q8) {
            asm volatile("" : "+v"(k));   // (places found here: kept over the items, a few of them spill)
            const int wide = row_codes(d), kc = min(k, wide - 8);
#pragma unroll
            for (int u = 0; u < kEach; ++u) {
                const size_t row = (size_t)max(id_of(u), 0);
                const uint2 c = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(r.x) + row * wide + kc);
                v[u] = make_uint4(c.x, c.y, r.scales[row * (wide / kRowBlock) + kc / kRowBlock], 0u);
            }
        } else {
            // 16 bytes, from any multiple of 8; at a row's end its last 16,
            // whose upper half counts where d is no multiple of 8.  Rows of
            // four entries: 16 bytes from the row on, or for the last row of
            // all from the one before.
            typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(8)));
            const int kc = max(min(k, d - 8), 0);
#pragma unroll
            for (int u = 0; u < kEach; ++u) {
                const uint16_t *x = static_cast<const uint16_t *>(r.x) + (size_t)min(max(id_of(u), 0), r.last) * d;
                const u32x4u q = *reinterpret_cast<const u32x4u *>(x + kc);
                v[u] = make_uint4(q[0], q[1], q[2], q[3]);
            }
        }
    }
    // The eight entries of piece u (bf16).  ONE: entry d is 1.
    template <bool ONE>
    __device__ __forceinline__ uint4 piece(const Rows &r, int k0, int d, int u) const {
        const int k = k0 + col();
        const bool full = k + 8 <= d, half = k + 4 == d, row_in = id_of(u) >= 0;
        uint4 p = v[u];
        if constexpr (Q8) {
            p = eight_of_codes(make_uint2(p.x, p.y), p.z);
            p = make_uint4(p.x, p.y, full ? p.z : 0u, full ? p.w : 0u);
        } else {
            const bool low = full || (d < 8 && id_of(u) <= r.last);
            p = make_uint4(low ? p.x : p.z, low ? p.y : p.w, full ? p.z : 0u, full ? p.w : 0u);
        }
        const bool in = row_in && (full || half);
        p = make_uint4(in ? p.x : 0u, in ? p.y : 0u, in ? p.z : 0u, in ? p.w : 0u);
        if constexpr (ONE) {
            p.x = row_in && k == d ? 0x3F80u : p.x;
            p.z = row_in && half ? 0x3F80u : p.z;
        }
        return p;
    }
    template <bool ONE>
    __device__ __forceinline__ void store(const Rows &r, int k0, int d, uint16_t *to, int stride) const {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const uint4 p = piece<ONE>(r, k0, d, u);
            if (col() < stride) *reinterpret_cast<uint4 *>(to + (kRows * w + row(u)) * stride + col()) = p;
        }
    }
    // Of the eight, infinities and NaN: bits 0x8000 of the halves.
    static __device__ __forceinline__ uint32_t not_finite(const uint4 &p) {
        auto over = [](uint32_t x) { return (x & 0x7FFF7FFFu) + 0x00800080u; };
        return over(p.x) | over(p.y) | over(p.z) | over(p.w);
    }
    // The same, but rows with an infinity or NaN are stored as zeros, and told of:
    // bit u is row kRows w + u.
    template <bool ONE>
    __device__ __forceinline__ uint32_t store_finite(const Rows &r, int k0, int d, uint16_t *to, int stride) const {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
        uint32_t any = 0;
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const uint4 p = piece<ONE>(r, k0, d, u);
            any |= not_finite(p);
            if (col() < stride) *reinterpret_cast<uint4 *>(to + (kRows * w + row(u)) * stride + col()) = p;
        }
        uint32_t bad = 0;
        if (__ballot((any & 0x80008000u) != 0) == 0) return bad;
        // (rarely: from LDS, row by row.  The asm keeps what only this needs out of
        // the registers of the loop around it)
        int at = 8 * lane, zero = 0;
        asm volatile("" : "+v"(at), "+v"(zero));
#pragma unroll 1
        for (int u = 0; u < kRows; ++u) {
            uint16_t *p = to + (kRows * w + u) * stride + at;
            const bool hit = at < min(stride, COLS) && (not_finite(*reinterpret_cast<const uint4 *>(p)) & 0x80008000u) != 0;
            if (__ballot(hit) == 0) continue;
            bad |= 1u << u;
            if (at < stride) *reinterpret_cast<uint4 *>(p) = make_uint4(zero, zero, zero, zero);
        }
        return bad;
    }
};

// A label's gradient and where each post's cell (i, i) would be in it: the
// caller's [B][N1][N1], or the compact cells of the label
// (KernelPlan::post_cells).
struct Grad {
    const float *g;
    const int64_t *cells;
};
// G of rows i in block `bi` and columns j in block `bj`: the cells of one
// sentence with i < j, zero elsewhere (other cells are not used).  Posts of a
// sentence are neighbours, so row r's cells are its n - i next columns.
// Wavefront w of NW takes kRows rows from kRows w on, a lane a column, so that
// rows are read along memory, what a row needs is scalar and rows of a lane are
// neighbours in G^T[j][i]; as bf16 hi and lo parts.
template <int NW>
struct Staged_grad {
    static constexpr int kRows = kBlk / NW;
    float v[kRows];
    uint32_t in;
    // What does not depend on the label: where a row's cell (i, i+1) is, and a
    // lane's place after it in bytes.  (Found anew for each label, the rows of 138
    // labels took 72 us and not 62.)
    struct Places {
        int64_t cell[kRows];
        uint32_t after[kRows], in;
    };
    static __device__ __forceinline__ Places places(const int64_t *cells, const int32_t *posts, int blk) {
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int at = lane - kRows * w - 1;
        Places p;
        p.in = 0;
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            p.cell[u] = constant(cells + (size_t)blk * kBlk + kRows * w + u) + 1;
            const bool ok = (uint32_t)(at - u) < (uint32_t)constant(posts + (size_t)blk * kPostRec + kBlk + kRows * w + u);
            p.in |= ok ? 1u << u : 0u;
            p.after[u] = ok ? 4u * (uint32_t)(at - u) : 0u;
        }
        return p;
    }
    __device__ __forceinline__ void load(const float *g, const Places &p) {
        in = p.in;
#pragma unroll
        for (int u = 0; u < kRows; ++u)
            v[u] = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(g + p.cell[u]) + p.after[u]);
    }
    __device__ __forceinline__ void load(const Grad &g, const int32_t *posts, int bi, int bj) {
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int32_t *rest = posts + (size_t)bi * kPostRec + kBlk + kRows * w;
        const int64_t *cell = g.cells + (size_t)bi * kBlk + kRows * w;
        int n[kRows];
        int64_t c[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) n[u] = constant(rest + u);
#pragma unroll
        for (int u = 0; u < kRows; ++u) c[u] = constant(cell + u);
        const int at = kBlk * (bj - bi) + lane - kRows * w - 1;   // j - i - 1 of row kRows w
        in = 0;
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const bool ok = (uint32_t)(at - u) < (uint32_t)n[u];
            in |= ok ? 1u << u : 0u;
            v[u] = (g.g + c[u] + 1)[ok ? at - u : 0];   // (else cell (i, i+1), which exists)
        }
    }
    // hi, lo: [64][kGS] each
    __device__ __forceinline__ void store(uint16_t *hi, uint16_t *lo) const {
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int q = 0; q < kRows / 4; ++q) {
            float x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = in >> (4 * q + u) & 1u ? v[4 * q + u] : 0.f;
            uint2 h, l;
            parts(x[0], x[1], h.x, l.x);
            parts(x[2], x[3], h.y, l.y);
            *reinterpret_cast<uint2 *>(hi + lane * kGS + kRows * w + 4 * q) = h;
            *reinterpret_cast<uint2 *>(lo + lane * kGS + kRows * w + 4 * q) = l;
        }
    }
};
// Operands of the staged G^T with K numbered as a wavefront holds the other
// operand after a product: a lane's eight are posts 32 p + 4 lg .. +3 and the
// four that come 16 later.  Posts 16 r .. +15: rows j with K over i, or (ROWS_I)
// rows i with K over j.
template <bool ROWS_I>
__device__ __forceinline__ bf16x8 grad_frag(const uint16_t *gt, int r, int p, int lr, int lg) {
    if constexpr (ROWS_I) {
        const uint16_t *q = gt + (32 * p + 4 * lg + (lr >> 2)) * kGS + 16 * r + 4 * (lr & 3);
        return frag_rows(q, q + 16 * kGS);
    } else {
        const uint16_t *q = gt + (16 * r + lr) * kGS + 32 * p + 4 * lg;
        const uint2 x = *reinterpret_cast<const uint2 *>(q), y = *reinterpret_cast<const uint2 *>(q + 16);
        return __builtin_bit_cast(bf16x8, make_uint4(x.x, x.y, y.x, y.y));
    }
}
// Whether that part of a block's product with itself can be other than zero
// (i < j).
template <bool ROWS_I>
__device__ __forceinline__ constexpr bool grad_part(int r, int p) {
    return ROWS_I ? 32 * p + 31 > 16 * r : 32 * p < 16 * r + 15;
}

// W's fragments for the dense products, from W transposed as the scorer takes
// it (w[l][c][a], row stride ldw), zero past its d x (d+1) entries: per label,
// side, step of 32 of K and block of 16 output columns, 64 lanes' eight
// entries.  Side 0 (dR^l): column a, K over c; side 1 (dR^r): column c, K over a.
__global__ __launch_bounds__(256) void bwd_weights_kernel(const uint16_t *__restrict__ w, int d, int ldw, int dp, int64_t pieces,
                                                          uint16_t *__restrict__ out) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= pieces) return;
    const int lane = (int)(t & 63), nb = dp / 16;
    const int64_t q = t >> 6;
    const int col = 16 * (int)(q % nb) + (lane & 15), k = 32 * (int)(q / nb % (dp / 32)) + 8 * (lane >> 4);
    const int side = (int)(q / nb / (dp / 32) & 1);
    const uint16_t *wl = w + (size_t)(q / nb / (dp / 32) >> 1) * d * ldw;
    uint16_t v[8];
    if (side) {   // (a wavefront's pieces are of one side.  Fours of a row are inside it up to entry d's)
        const bool in = col < d;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int a = k + 4 * h;
            const uint2 x = in && a <= d ? *reinterpret_cast<const uint2 *>(wl + (size_t)col * ldw + a) : make_uint2(0u, 0u);
            const uint32_t words[2] = {x.x, x.y};
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * h + e] = a + e <= d ? (uint16_t)(words[e >> 1] >> (16 * (e & 1))) : (uint16_t)0;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k + e < d && col <= d ? wl[(size_t)(k + e) * ldw + col] : (uint16_t)0;
    }
    *reinterpret_cast<uint4 *>(out + 8 * t) =
        make_uint4(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16, v[4] | (uint32_t)v[5] << 16,
                   v[6] | (uint32_t)v[7] << 16);
}

// Labelled gradients [cell][L] to [L][cell], cells compact: a wavefront takes
// a row of cells (i, i+1..n) and 64 labels, 32 cells at a time through LDS.
constexpr int kTrCells = 32;
__global__ __launch_bounds__(256) void bwd_compact_kernel(const int32_t *__restrict__ posts,
                                                          const int64_t *__restrict__ post_cells,
                                                          const int64_t *__restrict__ square_cells, int L, int64_t cells,
                                                          const float *__restrict__ g, float *__restrict__ out) {
    __shared__ float tile[4][kTrCells][65];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = (int)blockIdx.x * 4 + wave, l0 = (int)blockIdx.y * 64;
    const int32_t *rec = posts + (size_t)(row / kBlk) * kPostRec + row % kBlk;
    const int id = rec[0];
    if (id < 0) return;   // (wavefronts share nothing)
    const int n = rec[kBlk];   // cells of the row
    const int ls = min(64, L - l0);
    const float *src = g + square_cells[row] * L + l0 + min(lane, ls - 1);
    float *to = out + (int64_t)l0 * cells + post_cells[row];
    const int c = lane % kTrCells, lhalf = lane / kTrCells;
    for (int j0 = 1; j0 <= n; j0 += kTrCells) {
        const int m = min(kTrCells, n + 1 - j0);
        // eight loads in flight, the last cell's again at the end: no branch
        for (int x = 0; x < m; x += 8) {
            float v[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) v[t] = src[(int64_t)(j0 + min(x + t, m - 1)) * L];
#pragma unroll
            for (int t = 0; t < 8; ++t) tile[wave][x + t][lane] = v[t];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (c < m)
            for (int l = lhalf; l < ls; l += 2) to[(int64_t)l * cells + j0 + c] = tile[wave][c][l];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

struct BwdArgs {
    const int32_t *posts;
    const int64_t *post_cells;
    int n_posts, blk0, blks;            // the batch's blocks, and those of this launch
    int d, L, per_group;                // per_group: labels of a group
    Rows rl, rr;
    const uint16_t *wf;                 // bwd_weights_kernel's fragments
    const float *g;
    int64_t cells;                      // floats between the labels of a compact gradient
    uint16_t *out[2];                   // dR^l, dR^r
    float *part;                        // [label groups][2][posts][DP]: partial sums, or NULL
    int zs;                             // items that share blocks' output columns
    int items, side0;                   // items of a side; the first grid.y's side
};
// An item: its block, labels and column share.
struct Item {
    int blk, l0, l1, cz, grp;
};
__device__ __forceinline__ Item item_of(const BwdArgs &a, int it) {
    const int q = it / a.blks;
    Item x;
    x.blk = a.blk0 + it - q * a.blks;
    x.cz = q % a.zs;
    x.grp = q / a.zs;
    x.l0 = x.grp * a.per_group;
    x.l1 = min(x.l0 + a.per_group, a.L);
    return x;
}
__device__ __forceinline__ const uint16_t *weight_frags(const BwdArgs &a, int l, int side, int dp, int col0) {
    return a.wf + ((((size_t)l * 2 + side) * (dp / 32)) * (dp / 16) + col0) * 512 + 8 * (threadIdx.x & 63);
}
// Of x and y in the four 16-lane rows of a wavefront, x0 x1 x2 x3 and y0 y1 y2
// y3: (x0 x2 y0 y2, x1 x3 y1 y3).
__device__ __forceinline__ uint2 trade(uint32_t x, uint32_t y) {
    const auto h = __builtin_amdgcn_permlane32_swap(x, y, false, false);         // x0 x1 y0 y1, x2 x3 y2 y3
    const auto q = __builtin_amdgcn_permlane16_swap(h[0], h[1], false, false);
    return make_uint2(q[0], q[1]);
}
// A lane's posts 16 r + lr of a block (all before the first store, which a later
// load would wait for).
struct Row_ids {
    int id[4];
    __device__ __forceinline__ void load(const BwdArgs &a, int blk) {
#pragma unroll
        for (int r = 0; r < 4; ++r) id[r] = a.posts[(size_t)blk * kPostRec + 16 * r + (int)(threadIdx.x & 15)];
    }
};
// o[c]: columns 16 (col0 + c) + 4 lg .. +3 of post 16 r + lr of block blk, whose
// id is `id`.  GROUPS: there may be label groups, whose sums are partial.
template <int CB, int SIDE, bool GROUPS>
__device__ __forceinline__ void store_rows(const BwdArgs &a, const f32x4 (&o)[CB], int id, int blk, int r, int grp, int col0,
                                           int dp) {
    const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
    if (id < 0) return;   // (the four lanes of a post alike)
    if (GROUPS && a.part != nullptr) {
        float *row = a.part + (((size_t)grp * 2 + SIDE) * a.n_posts * kBlk + kBlk * blk + 16 * r + lr) * dp;
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            const int col = 16 * (col0 + c) + 4 * lg;
            if (col < a.d) *reinterpret_cast<f32x4 *>(row + col) = o[c];
        }
        return;
    }
    // Two column blocks at a time: the four lanes of a post exchange their
    // fours, so that each has eight neighbours and a store writes 64 bytes of a
    // post's row.
    typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(8)));
    uint16_t *row = a.out[SIDE] + (size_t)id * a.d;
#pragma unroll
    for (int c = 0; c + 1 < CB; c += 2) {
        const uint2 x = __builtin_bit_cast(uint2, __builtin_convertvector(o[c], bf16x4));
        const uint2 y = __builtin_bit_cast(uint2, __builtin_convertvector(o[c + 1], bf16x4));
        const uint2 px = trade(x.x, y.x), py = trade(x.y, y.y);
        const int col = 16 * (col0 + c) + 8 * lg;
        if (col + 8 <= a.d) *reinterpret_cast<u32x4u *>(row + col) = u32x4u{px.x, py.x, px.y, py.y};
        else if (col < a.d) *reinterpret_cast<uint2 *>(row + col) = make_uint2(px.x, py.x);
    }
    if constexpr (CB % 2 != 0) {
        const int col = 16 * (col0 + CB - 1) + 4 * lg;
        if (col < a.d) *reinterpret_cast<bf16x4 *>(row + col) = __builtin_convertvector(o[CB - 1], bf16x4);
    }
}

// dR^l (side 0) and dR^r (side 1) of a block that holds whole sentences, as
// G (R^r W^T) and G^T ([R^l ; 1] W): V = R W first, whose K runs along rows of
// R, and W's fragments come straight from L2 in the order of the lanes.  A
// wavefront holds V of its 16 CB columns for all 64 posts, which is the layout
// of the second product's operand when K is numbered as in grad_frag: V, as
// two bf16 parts, never leaves the registers.  (As (G R) W^T, whose inner
// product goes through LDS, 5,000 sentences at d = 500 took 252 us, this way
// 207: 0.63e15 operations a second.)
//
// Two workgroups a CU (at d = 500 they fill its LDS): one's staging and stores
// run beside the other's products.  With 128 posts a workgroup and one on a CU,
// W came from L2 half as often, but 210 us.  R and G of a workgroup's next
// block are on their way to registers from the end of the dense product on.
// DP = 128 NB columns, 16 NW CB of them a workgroup.

// Row stride of R: past d, and an odd multiple of 16 bytes (16-byte operands of
// sixteen rows in different banks).  K runs past it into the next row (or G),
// where W's fragments are zero.
__host__ __device__ inline int row_stride(int d) { return (d / 8 + 1) * 8 + (d / 8 % 2 != 0 ? 8 : 0); }
template <bool COMPACT>
inline int posts_lds(int d) {
    return 2 * (kBlk * row_stride(d) + (COMPACT ? 2 : 1) * 2 * kBlk * kGS);
}

template <int NB, int NW, int CB, bool Q8, bool COMPACT, int SIDE>
__device__ __forceinline__ void bwd_posts(const BwdArgs &a, char *smem) {
    constexpr int DP = 128 * NB;
    constexpr bool ONE = SIDE == 1, ROWS_I = SIDE == 0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 15, lg = lane >> 4, RS = row_stride(a.d);
    uint16_t *R = reinterpret_cast<uint16_t *>(smem);   // [64][RS]
    uint16_t *G = R + kBlk * RS;                        // [COMPACT ? 2 : 1][2][64][kGS]: G^T, hi and lo
    const int ksteps = (a.d + 32) / 32;   // K of the dense product: d + 1 at most
    const Rows rows = SIDE == 0 ? a.rr : a.rl;

    constexpr bool AHEAD = CB <= 2 || COMPACT;   // (R of the next block beside V, in registers)
    Staged<DP, NW, Q8> sr;
    Staged_grad<NW> sg;
    auto load_r = [&](int blk) { sr.load(rows, a.posts + (size_t)blk * kPostRec, 0, a.d); };
    auto load_grad = [&](int blk, int l) {
        sg.load(Grad{a.g + (COMPACT ? l * a.cells : 0), a.post_cells}, a.posts, blk, blk);
    };
    f32x4 v[4][CB];
    // V = R W_l
    auto dense = [&](int l, int col0) {
        const uint16_t *wf = weight_frags(a, l, SIDE, DP, col0);
        const uint16_t *p = R + lr * RS + 8 * lg;
        bf16x8 wv[2][CB];   // two steps of W
#pragma unroll
        for (int c = 0; c < CB; ++c) wv[0][c] = frag(wf + (size_t)c * 512);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < CB; ++c) v[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto step = [&](int ks, bf16x8 (&now)[CB], bf16x8 (&then)[CB]) {
            const int kn = min(ks + 1, ksteps - 1);
#pragma unroll
            for (int c = 0; c < CB; ++c) then[c] = frag(wf + ((size_t)kn * (DP / 16) + c) * 512);
            bf16x8 pv = frag(p + 32 * ks);
            __builtin_amdgcn_sched_barrier(0);   // (left alone, they are issued where they are waited for)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                bf16x8 pn = pv;
                if (r + 1 < 4) {
                    int at = 16 * (r + 1) * RS + 32 * ks;
                    asm("" : "+s"(at));   // (a scalar: addresses kept for every r spill)
                    pn = frag(p + at);
                }
#pragma unroll
                for (int c = 0; c < CB; ++c) v[r][c] = mfma(pv, now[c], v[r][c]);
                pv = pn;
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        int ks = 0;
        for (; ks + 1 < ksteps; ks += 2) {
            step(ks, wv[0], wv[1]);
            step(ks + 1, wv[1], wv[0]);
        }
        if (ks < ksteps) step(ks, wv[0], wv[1]);
    };
    bf16x8 vh[2][CB], vl[2][CB];
    auto split_v = [&]() {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int c = 0; c < CB; ++c) two_parts(v[2 * p][c], v[2 * p + 1][c], vh[p][c], vl[p][c]);
    };
    // o += V^T G, posts 16 r .. +15
    auto second = [&](int r, const uint16_t *g, f32x4 (&o)[CB]) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
            if (grad_part<ROWS_I>(r, p)) {
                const bf16x8 gh = grad_frag<ROWS_I>(g, r, p, lr, lg), gl = grad_frag<ROWS_I>(g + kBlk * kGS, r, p, lr, lg);
#pragma unroll
                for (int c = 0; c < CB; ++c) o[c] = mfma(vh[p][c], gh, o[c]);
#pragma unroll
                for (int c = 0; c < CB; ++c) o[c] = mfma(vh[p][c], gl, o[c]);
#pragma unroll
                for (int c = 0; c < CB; ++c) o[c] = mfma(vl[p][c], gh, o[c]);
            }
    };
    auto clear = [](f32x4 (&o)[CB]) {
#pragma unroll
        for (int c = 0; c < CB; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    };

    // A representation that is not finite.  Its row of R is staged as zeros (times
    // a zero of G or W it would be NaN in the rows of other sentences), and the
    // rows of its own sentence become NaN through G: row 63 of G^T (ROWS_I) or
    // column 31 meet each of them in a part that is multiplied, and a V that is
    // finite (they are past the 24 entries that R's last row runs into).  Which
    // rows these are goes round in the padding of G's rows.
    static_assert(kGS - kBlk >= 2 && kBlk / NW <= 16);
    uint32_t *const bad_rows = reinterpret_cast<uint32_t *>(G + kBlk);   // wavefront w's: word w kGS / 2
    auto poison = [&](int blk, uint32_t mine) {   // mine: lane w's word (every wavefront alike)
        if (__ballot(mine != 0) == 0) return;
        const int32_t *rest = a.posts + (size_t)blk * kPostRec + kBlk;
        auto is_bad = [&](int post) { return bad_rows[post / (kBlk / NW) * (kGS / 2)] >> (post % (kBlk / NW)) & 1u; };
        int post = threadIdx.x;
        asm volatile("" : "+v"(post));
        if (post < kBlk && rest[post - kBlk] >= 0) {
            int first = post, last = post;
            while (first > 0 && rest[first - 1] > 0) --first;   // (a sentence's last post has no cells)
            while (rest[last] > 0) ++last;
            uint32_t any = 0;
            for (int k = first; k <= last; ++k) any |= is_bad(k);
            if (any) G[ROWS_I ? (kBlk - 1) * kGS + post : post * kGS + 31] = 0x7FC0;
        }
        __syncthreads();
    };
    auto bad_word = [&]() { return lane < NW ? bad_rows[lane * (kGS / 2)] : 0u; };

    int it = blockIdx.x;
    if (it >= a.items) return;
    Item x = item_of(a, it);
    auto load_item = [&](const Item &y) {
        load_r(y.blk);
        load_grad(y.blk, y.l0);
    };
    if constexpr (AHEAD) load_item(x);
    for (;;) {
        if constexpr (!AHEAD) load_item(x);
        const int next_it = it + gridDim.x;
        const Item nx = item_of(a, min(next_it, a.items - 1));
        const int col0 = (x.cz * NW + wave) * CB;   // the wavefront's first column block
        const uint32_t bad = sr.template store_finite<ONE>(rows, 0, a.d, R, RS);
        if (lane == 0) bad_rows[wave * (kGS / 2)] = bad;
        sg.store(G, G + kBlk * kGS);
        if constexpr (COMPACT) {
            f32x4 o[4][CB];
#pragma unroll
            for (int r = 0; r < 4; ++r) clear(o[r]);
            const typename Staged_grad<NW>::Places at = sg.places(a.post_cells, a.posts, x.blk);
            sg.load(a.g + min(x.l0 + 1, x.l1 - 1) * a.cells, at);
            __syncthreads();
            poison(x.blk, bad_word());
            for (int l = x.l0; l < x.l1; ++l) {
                uint16_t *now = G + ((l - x.l0) & 1) * 2 * kBlk * kGS, *then = G + ((l - x.l0 + 1) & 1) * 2 * kBlk * kGS;
                sg.store(then, then + kBlk * kGS);   // (its readers are a barrier behind)
                sg.load(a.g + min(l + 2, x.l1 - 1) * a.cells, at);
                __builtin_amdgcn_sched_barrier(0);
                dense(l, col0);
                split_v();
                if constexpr (CB > 1) __builtin_amdgcn_sched_barrier(0);   // (or a few registers spill)
#pragma unroll
                for (int r = 0; r < 4; ++r) second(r, now, o[r]);
                __syncthreads();
            }
            load_item(nx);
            __builtin_amdgcn_sched_barrier(0);
            Row_ids ids;
            ids.load(a, x.blk);
#pragma unroll
            for (int r = 0; r < 4; ++r) store_rows<CB, SIDE, COMPACT>(a, o[r], ids.id[r], x.blk, r, x.grp, col0, DP);
        } else {
            __syncthreads();
            poison(x.blk, bad_word());
            dense(0, col0);
            split_v();
            __builtin_amdgcn_sched_barrier(0);   // (the registers of V hold the next R)
            Row_ids ids;
            ids.load(a, x.blk);
            if constexpr (AHEAD) load_item(nx);   // (past the last item, that one's again)
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                f32x4 o[CB];
                clear(o);
                second(r, G, o);
                store_rows<CB, SIDE, COMPACT>(a, o, ids.id[r], x.blk, r, x.grp, col0, DP);
            }
            __syncthreads();   // the readers of R and G are done
        }
        if (next_it >= a.items) break;
        it = next_it;
        x = nx;
    }
}

// (four wavefronts a SIMD, fewer with sums over labels beside V)
constexpr int posts_waves(int cb, bool compact) { return !compact || cb == 1 ? 4 : cb == 2 ? 3 : 2; }
template <int NB, int NW, int CB, bool Q8, bool COMPACT>
__global__ __launch_bounds__(64 * NW, posts_waves(CB, COMPACT)) void bwd_posts_kernel(BwdArgs a) {
    extern __shared__ __align__(16) char smem[];
    if (blockIdx.y + a.side0 == 0) bwd_posts<NB, NW, CB, Q8, COMPACT, 0>(a, smem);
    else bwd_posts<NB, NW, CB, Q8, COMPACT, 1>(a, smem);
}

// The same of blocks of a sentence that has more than one, as (G R^r) W^T and
// (G^T [R^l ; 1]) W: a block of posts meets every block on its side of the
// diagonal, and only the product with G is repeated for them, not the dense
// one.  U = G R (or X) goes into LDS as two bf16 parts, the first where R was
// (its columns are in registers until every wavefront has read R), 64 x DP; R and G of the next
// block are in flight in registers during this one's products.  CB: 16-column
// blocks of the output a wavefront.
constexpr int kLongWaves = 8;
template <int NB>
struct LongShape {
    static constexpr int kDP = 128 * NB, kPS = kDP + 8;
    static constexpr int kLds = 2 * (2 * kBlk * kPS + 2 * kBlk * kGS);
};

template <int NB, int CB, bool Q8, bool COMPACT, int SIDE>
__device__ __forceinline__ void bwd_long(const BwdArgs &a, char *smem) {
    typedef LongShape<NB> S;
    constexpr int DP = S::kDP, PS = S::kPS;
    constexpr bool ONE = SIDE == 1, ROWS_I = SIDE == 0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 15, lg = lane >> 4;
    uint16_t *P = reinterpret_cast<uint16_t *>(smem);       // [2][64][PS]: R, then the parts of U or X
    uint16_t *Gh = P + 2 * kBlk * PS, *Gl = Gh + kBlk * kGS;
    const int ksteps = (a.d + 32) / 32;
    const Rows rows = SIDE == 0 ? a.rr : a.rl;

    // A block's partners: side 0 itself and those after it, side 1 those before it and itself.
    auto first_of = [&](int blk) { return SIDE == 0 ? blk : constant(a.posts + (size_t)blk * kPostRec + 2 * kBlk); };
    auto last_of = [&](int blk) { return SIDE == 0 ? constant(a.posts + (size_t)blk * kPostRec + 2 * kBlk + 1) : blk; };
    Staged<DP, kLongWaves, Q8> sr;
    Staged_grad<kLongWaves> sg;
    auto load_step = [&](int l, int blk, int q) {
        sg.load(Grad{a.g + (COMPACT ? l * a.cells : 0), a.post_cells}, a.posts, SIDE == 0 ? blk : q, SIDE == 0 ? q : blk);
        sr.load(rows, a.posts + (size_t)q * kPostRec, 0, a.d);
    };

    const int it = blockIdx.x;
    if (it >= a.items) return;
    const Item x = item_of(a, it);
    const int q0 = first_of(x.blk), q1 = last_of(x.blk), col0 = (x.cz * kLongWaves + wave) * CB;
    load_step(x.l0, x.blk, q0);
    f32x4 acc[4][CB];
    for (int l = x.l0;;) {   // (one label, l = 0, unless COMPACT)
        f32x4 u[NB][4];
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) u[c][r] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int q = q0; q <= q1; ++q) {
            __syncthreads();   // the readers of what is stored next are done
            sr.template store<ONE>(rows, 0, a.d, P, PS);
            sg.store(Gh, Gl);
            // the next partner, or the first one for the next label
            load_step(COMPACT ? min(q < q1 ? l : l + 1, x.l1 - 1) : l, x.blk, q < q1 ? q + 1 : q0);
            __syncthreads();
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                bf16x8 rf[NB];
                const uint16_t *at = P + (32 * p + 4 * lg + (lr >> 2)) * PS + 16 * wave * NB + 4 * (lr & 3);
#pragma unroll
                for (int c = 0; c < NB; ++c) rf[c] = frag_rows(at + 16 * c, at + 16 * PS + 16 * c);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (grad_part<ROWS_I>(r, p) || q != x.blk) {
                        const bf16x8 gh = grad_frag<ROWS_I>(Gh, r, p, lr, lg), gl = grad_frag<ROWS_I>(Gl, r, p, lr, lg);
#pragma unroll
                        for (int c = 0; c < NB; ++c) {
                            u[c][r] = mfma(rf[c], gh, u[c][r]);
                            u[c][r] = mfma(rf[c], gl, u[c][r]);
                        }
                        if constexpr (COMPACT && CB == 4) __builtin_amdgcn_sched_barrier(0);   // (or registers spill)
                    }
            }
        }
        __syncthreads();   // R's readers are done
        // u[c][r]: columns 16 (wave NB + c) + 4 lg .. +3 of post 16 r + lr
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                uint2 h, l;
                parts(u[c][r][0], u[c][r][1], h.x, l.x);
                parts(u[c][r][2], u[c][r][3], h.y, l.y);
                uint16_t *at = P + (16 * r + lr) * PS + 16 * (wave * NB + c) + 4 * lg;
                *reinterpret_cast<uint2 *>(at) = h;
                *reinterpret_cast<uint2 *>(at + kBlk * PS) = l;
            }
        __syncthreads();

        if (!COMPACT || l == x.l0)
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
        const uint16_t *wf = weight_frags(a, l, SIDE, DP, col0), *prow = P + lr * PS + 8 * lg;
        for (int ks = 0; ks < ksteps; ++ks) {
            bf16x8 wv[CB];
#pragma unroll
            for (int c = 0; c < CB; ++c) wv[c] = frag(wf + ((size_t)ks * (DP / 16) + c) * 512);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bf16x8 ph = frag(prow + 16 * r * PS + 32 * ks), pl = frag(prow + (kBlk + 16 * r) * PS + 32 * ks);
#pragma unroll
                for (int c = 0; c < CB; ++c) acc[r][c] = mfma(wv[c], ph, acc[r][c]);
#pragma unroll
                for (int c = 0; c < CB; ++c) acc[r][c] = mfma(wv[c], pl, acc[r][c]);
            }
        }
        if (!COMPACT || ++l >= x.l1) break;
    }
    Row_ids ids;
    ids.load(a, x.blk);
#pragma unroll
    for (int r = 0; r < 4; ++r) store_rows<CB, SIDE, COMPACT>(a, acc[r], ids.id[r], x.blk, r, x.grp, col0, DP);
}

template <int NB, int CB, bool Q8, bool COMPACT>
__global__ __launch_bounds__(64 * kLongWaves) void bwd_long_kernel(BwdArgs a) {
    extern __shared__ __align__(16) char smem[];
    if (blockIdx.y + a.side0 == 0) bwd_long<NB, CB, Q8, COMPACT, 0>(a, smem);
    else bwd_long<NB, CB, Q8, COMPACT, 1>(a, smem);
}

// The label groups' partial sums of dR^l and dR^r, added in their order: a
// thread per post and four columns.
__global__ __launch_bounds__(256) void bwd_join_rows_kernel(const int32_t *__restrict__ posts, int n_posts, int d, int dp,
                                                            int groups, const float *__restrict__ part,
                                                            uint16_t *__restrict__ out_l, uint16_t *__restrict__ out_r, int side0) {
    const int side = (int)blockIdx.y + side0, per = d / 4;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= (int64_t)n_posts * kBlk * per) return;
    const int64_t slot = t / per;
    const int col = 4 * (int)(t - slot * per), id = posts[slot / kBlk * kPostRec + slot % kBlk];
    if (id < 0) return;
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int q = 0; q < groups; ++q)
        s += *reinterpret_cast<const f32x4 *>(part + (((size_t)q * 2 + side) * n_posts * kBlk + slot) * dp + col);
    *reinterpret_cast<bf16x4 *>((side ? out_r : out_l) + (size_t)id * d + col) = __builtin_convertvector(s, bf16x4);
}

// dW of one label, a tile of 16 AB columns a by 16 T NW rows c, over a share of
// the blocks of posts: a wavefront holds U = G R^r of its 16 T columns c in
// registers, whose layout is that of the second product's operand when K is
// numbered as in grad_frag, as hi and lo parts.  (dW is 3.1e-6 off for the two
// pairs of parts.  Three of each, all 24 bits of G and U, give 9e-8, and take a
// call of 5,000 sentences at d = 500 9% and one of 200 5% longer, for a gradient
// whose representations have 8 bits.)  A step is a block and one of
// its partners: U grows by their product, then R^r and G of the next step (and
// [R^l ; 1] of the next block, into the other of its two places) go from
// registers to LDS and those of the step after it start on their way, and
// [R^l ; 1]^T U of a block that has met all its partners is added.
//
// The tiles of a share read the same posts: they are neighbours on one XCD, so
// that a post's rows come from HBM once.
//
// 5,000 sentences at d = 500: 252 us, of which the matrix instructions take 90
// (U's two parts and G's make the products twice as many).  The rest is what
// two wavefronts a SIMD do not hide: staging's and splitting's arithmetic and
// LDS reads between the barriers.  Two workgroups of four wavefronts a CU, tiles
// of 256 x 128, whose phases drift apart, took 284 (then against 250): [R^l ; 1] is
// staged twice.
struct WeightArgs {
    const int32_t *posts;
    const int64_t *post_cells;
    int n_posts, d, ldw, L, splits, tiles_a, tiles;
    Rows rl, rr;
    const float *g;
    int64_t cells;
    float *out;   // splits = 1: dW [L][d][ldw]; else partial sums [splits][L][d][d + 4]
};
template <int AB, int T, int NW>
struct WeightShape {
    static constexpr int kA = 16 * AB, kC = 16 * T * NW, kAS = kA + 8, kCS = kC + 8;
    static constexpr int kLds = 2 * kBlk * (2 * kAS + kCS + 2 * kGS);
};
constexpr int kXcds = 8;

template <int AB, int T, int NW, bool Q8, bool COMPACT>
__global__ __launch_bounds__(64 * NW, 2) void bwd_weight_kernel(WeightArgs a) {
    extern __shared__ __align__(16) char smem[];
    typedef WeightShape<AB, T, NW> S;
    constexpr int TA = S::kA, TC = S::kC, AS = S::kAS, CS = S::kCS;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 15, lg = lane >> 4;
    uint16_t *Ra = reinterpret_cast<uint16_t *>(smem), *Rc = Ra + 2 * kBlk * AS;
    uint16_t *Gh = Rc + kBlk * CS, *Gl = Gh + kBlk * kGS;
    // workgroup b runs on XCD b mod 8: a (share, label)'s tiles side by side there
    const int per = kXcds * a.tiles, unit = (int)blockIdx.x / per * kXcds + (int)blockIdx.x % kXcds;
    const int tile = (int)blockIdx.x % per / kXcds;
    if (unit >= a.splits * a.L) return;
    const int split = unit / a.L, l = unit - split * a.L;
    const int a0 = TA * (tile % a.tiles_a), c0 = TC * (tile / a.tiles_a);
    const int b0 = (int)((int64_t)a.n_posts * split / a.splits), b1 = (int)((int64_t)a.n_posts * (split + 1) / a.splits);
    const Grad g{a.g + (COMPACT ? l * a.cells : 0), a.post_cells};

    f32x4 acc[AB][T];
#pragma unroll
    for (int x = 0; x < AB; ++x)
#pragma unroll
        for (int c = 0; c < T; ++c) acc[x][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    f32x4 u[4][T];
    auto clear_u = [&]() {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < T; ++c) u[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    clear_u();

    auto last_of = [&](int blk) { return constant(a.posts + (size_t)blk * kPostRec + 2 * kBlk + 1); };
    Staged<TA, NW, Q8> sa;
    Staged<TC, NW, Q8> sc;
    Staged_grad<NW> sg;
    auto post = [&](int blk) { return a.posts + (size_t)blk * kPostRec; };
    auto fetch = [&](int blk, int q) {
        sg.load(g, a.posts, blk, q);
        sc.load(a.rr, post(q), c0, a.d);
        if (q == blk) sa.load(a.rl, post(blk), a0, a.d);
    };
    auto stage = [&](int blk, int q) {
        sc.template store<false>(a.rr, c0, a.d, Rc, CS);
        if (q == blk) sa.template store<true>(a.rl, a0, a.d, Ra + (blk & 1) * kBlk * AS, AS);
        sg.store(Gh, Gl);
    };
    int blk = b0, q = b0, last = 0, nblk = b0, nq = b0;   // this step and the next
    auto advance = [&]() {
        if (nq < last) {
            ++nq;
        } else if (++nblk < b1) {
            nq = nblk;
            last = last_of(nblk);
        }
    };
    if (b0 < b1) {
        last = last_of(b0);
        fetch(b0, b0);
        stage(b0, b0);
        advance();
        if (nblk < b1) fetch(nblk, nq);
        __syncthreads();
    }
    while (blk < b1) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const uint16_t *at = Rc + (32 * p + 4 * lg + (lr >> 2)) * CS + 16 * wave * T + 4 * (lr & 3);
            bf16x8 rf[T];
#pragma unroll
            for (int c = 0; c < T; ++c) rf[c] = frag_rows(at + 16 * c, at + 16 * CS + 16 * c);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (grad_part<true>(r, p) || q != blk) {
                    const bf16x8 gh = grad_frag<true>(Gh, r, p, lr, lg), gl = grad_frag<true>(Gl, r, p, lr, lg);
#pragma unroll
                    for (int c = 0; c < T; ++c) u[r][c] = mfma(gh, rf[c], u[r][c]);
#pragma unroll
                    for (int c = 0; c < T; ++c) u[r][c] = mfma(gl, rf[c], u[r][c]);
                }
        }
        __syncthreads();   // the readers of R^r and G are done
        const bool whole = nblk != blk;   // the block has met all its partners
        const int nb = nblk, nqq = nq;
        if (nb < b1) {
            stage(nb, nqq);
            advance();
            if (nblk < b1) fetch(nblk, nq);
        }
        if (whole) {
#pragma unroll
            for (int kp = 0; kp < 2; ++kp) {
                bf16x8 hi[T], lo[T];
#pragma unroll
                for (int c = 0; c < T; ++c) two_parts(u[2 * kp][c], u[2 * kp + 1][c], hi[c], lo[c]);
                const uint16_t *p = Ra + (blk & 1) * kBlk * AS + (32 * kp + 4 * lg + (lr >> 2)) * AS + 4 * (lr & 3);
                bf16x8 af = frag_rows(p, p + 16 * AS);
#pragma unroll
                for (int x = 0; x < AB; ++x) {
                    bf16x8 an = af;
                    if (x + 1 < AB) an = frag_rows(p + 16 * (x + 1), p + 16 * AS + 16 * (x + 1));
#pragma unroll
                    for (int c = 0; c < T; ++c) acc[x][c] = mfma(af, hi[c], acc[x][c]);
#pragma unroll
                    for (int c = 0; c < T; ++c) acc[x][c] = mfma(af, lo[c], acc[x][c]);
                    af = an;
                }
            }
            clear_u();
        }
        __syncthreads();
        blk = nb;
        q = nqq;
    }

    // acc[x][c]: a = a0 + 16 x + 4 lg .. +3 of row c0 + 16 (wave T + c) + lr
    const bool whole = a.splits == 1;
    const int stride = whole ? a.ldw : a.d + 4;
    float *out = a.out + ((size_t)split * a.L + l) * a.d * stride;
#pragma unroll
    for (int c = 0; c < T; ++c) {
        const int row = c0 + 16 * (wave * T + c) + lr;
        if (row >= a.d) continue;
#pragma unroll
        for (int x = 0; x < AB; ++x) {
            const int col = a0 + 16 * x + 4 * lg;
            float *at = out + (size_t)row * stride + col;
            if (col < a.d || (!whole && col == a.d)) *reinterpret_cast<f32x4 *>(at) = acc[x][c];
            else if (col == a.d) *at = acc[x][c][0];
        }
    }
}

// The shares' partial sums of dW, added in their order: a thread per row c and
// four columns a.
__global__ __launch_bounds__(256) void bwd_join_weight_kernel(int d, int ldw, int64_t rows, int splits,
                                                              const float *__restrict__ part, float *__restrict__ out) {
    const int per = d / 4 + 1;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= rows * per) return;
    const int64_t row = t / per;
    const int col = 4 * (int)(t - row * per);
    const float *p = part + row * (d + 4) + col;
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int q = 0; q < splits; ++q) s += *reinterpret_cast<const f32x4 *>(p + (size_t)q * rows * (d + 4));
    float *at = out + row * ldw + col;
    if (col < d) *reinterpret_cast<f32x4 *>(at) = s;
    else *at = s[0];
}

// ---------------------------------------------------------------------------
// Launches.

inline int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

constexpr int kCus = 256, kLdsPerCu = 163840;

// How a call is cut up, and its workspace.
struct BwdPlan {
    int nb, dp;                     // DP = 128 nb
    bool few, few_long;             // few blocks (whole sentences, long ones): nb items share their columns
    int groups, per_group;          // label groups and labels of one
    bool wide;                      // dW in tiles of 256 x 256, else 128 x 128
    int tiles_a, tiles, splits;
    int64_t w_at, g_at, part_at, wpart_at, bytes;
};
BwdPlan bwd_plan(const KernelPlan &p, int64_t cells, int d, int L) {
    BwdPlan b{};
    b.nb = (d + 1 + 127) / 128;
    b.dp = 128 * b.nb;
    // (items for 3 workgroups a CU.  100 sentences, 138 labels, rows and the sums of
    // the groups: 139 us with items for 2, 120 with 3 or 4, 123 with 6, whose sums
    // cost more)
    b.groups = std::max(1, std::min(L, 3 * kCus / p.n_posts));
    b.per_group = (L + b.groups - 1) / b.groups;
    b.groups = (L + b.per_group - 1) / b.per_group;
    // (both sides' items, each times nb, are then at most two a CU, or one a CU of
    // the long kernel's.  One sentence of 25 words at d = 500: 8.5 us, 10.7 else;
    // three of 80 words 15.3, 17.8 else.  With twice the bound 200 sentences took
    // 22.2 and not 15, 5,000 with few long ones 48 for those and not 23: each of
    // nb items stages the block anew, and the long ones' repeat U.)
    b.few = (int64_t)(p.n_posts - p.n_long_posts) * b.groups * b.nb <= kCus;
    b.few_long = (int64_t)p.n_long_posts * b.groups * b.nb <= kCus / 2;
    // (a wide tile reads each row for half as many tiles: d = 500 250 us against
    // 398 of narrow ones for 5,000 sentences, 21.7 against 22.0 for 200; where one
    // narrow tile holds all it is the other way, d = 100 with 138 labels 70
    // against 200)
    b.wide = d + 1 > 128;
    const int tile = b.wide ? 256 : 128;
    b.tiles_a = (d + 1 + tile - 1) / tile;
    b.tiles = b.tiles_a * ((d + tile - 1) / tile);
    // (a share of two blocks at least: of one, 200 sentences at d = 500 take 10.3 us
    // for the sum of the shares and not 7.6, and dW no less)
    b.splits = (int)std::max<int64_t>(1, std::min<int64_t>((p.n_posts + 1) / 2, (b.wide ? 1 : 2) * kCus / ((int64_t)b.tiles * L)));
    int64_t at = 0;
    b.w_at = at;
    at += up256((int64_t)L * 2 * b.dp * b.dp * 2);
    b.g_at = at;
    if (L > 1) at += up256(cells * L * 4);
    b.part_at = at;
    if (b.groups > 1) at += up256((int64_t)b.groups * 2 * p.n_posts * kBlk * b.dp * 4);
    b.wpart_at = at;
    if (b.splits > 1) at += up256((int64_t)b.splits * L * d * (d + 4) * 4);
    b.bytes = at;
    return b;
}

// Every build of bwd_posts_kernel: nb, few, then NB, NW, CB; and of
// bwd_long_kernel: nb, few, NB, CB.
#define CRF_BWD_POSTS(F)                                                                            \
    F(1, false, 1, 4, 2) F(2, false, 2, 8, 2) F(3, false, 3, 8, 3) F(4, false, 4, 8, 4) F(1, true, 1, 8, 1) \
    F(2, true, 2, 8, 1) F(3, true, 3, 8, 1) F(4, true, 4, 8, 1)
#define CRF_BWD_LONG(F) \
    F(1, false, 1, 1) F(2, false, 2, 2) F(3, false, 3, 3) F(4, false, 4, 4) F(2, true, 2, 1) F(3, true, 3, 1) F(4, true, 4, 1)

template <int NB, int NW, int CB, bool Q8, bool COMPACT>
hipError_t launch_posts(BwdArgs a, int sides, int groups, hipStream_t stream) {
    a.zs = 8 * NB / (NW * CB);
    a.items = a.blks * a.zs * groups;
    const int lds = posts_lds<COMPACT>(a.d), regs = 4 * posts_waves(CB, COMPACT) / NW;   // workgroups a CU, by registers
    const int slots = std::max(1, std::min(regs, kLdsPerCu / lds)) * kCus / sides;
    hipLaunchKernelGGL((bwd_posts_kernel<NB, NW, CB, Q8, COMPACT>), dim3(std::min(a.items, slots), sides), dim3(64 * NW), lds,
                       stream, a);
    return hipGetLastError();
}
template <int NB, int CB, bool Q8, bool COMPACT>
hipError_t launch_long(BwdArgs a, int sides, int groups, hipStream_t stream) {
    a.zs = NB / CB;
    a.items = a.blks * a.zs * groups;
    hipLaunchKernelGGL((bwd_long_kernel<NB, CB, Q8, COMPACT>), dim3(a.items, sides), dim3(64 * kLongWaves), LongShape<NB>::kLds,
                       stream, a);
    return hipGetLastError();
}
template <bool Q8, bool COMPACT>
hipError_t launch_rows(const BwdPlan &b, BwdArgs a, int n_long, int sides, hipStream_t stream) {
    if (n_long > 0) {   // (the longest items first)
        a.blk0 = 0;
        a.blks = n_long;
        const bool few = b.few_long && b.nb > 1;
        hipError_t e = hipErrorInvalidValue;
#define CRF_LAUNCH(N, FEW, NB, CB) \
        if (b.nb == N && few == FEW) e = launch_long<NB, CB, Q8, COMPACT>(a, sides, b.groups, stream);
        CRF_BWD_LONG(CRF_LAUNCH)
#undef CRF_LAUNCH
        if (e != hipSuccess) return e;
    }
    a.blk0 = n_long;
    a.blks = a.n_posts - n_long;
    if (a.blks == 0) return hipSuccess;
#define CRF_LAUNCH(N, FEW, NB, NW, CB) \
    if (b.nb == N && b.few == FEW) return launch_posts<NB, NW, CB, Q8, COMPACT>(a, sides, b.groups, stream);
    CRF_BWD_POSTS(CRF_LAUNCH)
#undef CRF_LAUNCH
    return hipErrorInvalidValue;
}
template <bool Q8, bool COMPACT>
hipError_t launch_weight(const BwdPlan &b, const WeightArgs &a, hipStream_t stream) {
    const dim3 grid((unsigned)(((int64_t)a.splits * a.L + kXcds - 1) / kXcds * kXcds * b.tiles));
    if (b.wide)
        hipLaunchKernelGGL((bwd_weight_kernel<16, 2, 8, Q8, COMPACT>), grid, dim3(512), (WeightShape<16, 2, 8>::kLds), stream, a);
    else
        hipLaunchKernelGGL((bwd_weight_kernel<8, 2, 4, Q8, COMPACT>), grid, dim3(256), (WeightShape<8, 2, 4>::kLds), stream, a);
    return hipGetLastError();
}

template <bool Q8, bool COMPACT>
hipError_t set_attributes() {
    hipError_t e;
    auto set = [&](const void *f, int bytes) { return hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); };
#define CRF_SET(N, FEW, NB, NW, CB) \
    if ((e = set((const void *)bwd_posts_kernel<NB, NW, CB, Q8, COMPACT>, posts_lds<COMPACT>(kBiaMaxD))) != hipSuccess) return e;
    CRF_BWD_POSTS(CRF_SET)
#undef CRF_SET
#define CRF_SET(N, FEW, NB, CB) \
    if ((e = set((const void *)bwd_long_kernel<NB, CB, Q8, COMPACT>, LongShape<NB>::kLds)) != hipSuccess) return e;
    CRF_BWD_LONG(CRF_SET)
#undef CRF_SET
    if ((e = set((const void *)bwd_weight_kernel<16, 2, 8, Q8, COMPACT>, WeightShape<16, 2, 8>::kLds)) != hipSuccess ||
        (e = set((const void *)bwd_weight_kernel<8, 2, 4, Q8, COMPACT>, WeightShape<8, 2, 4>::kLds)) != hipSuccess)
        return e;
    return hipSuccess;
}

}  // namespace

int64_t biaffine_bwd_bytes(const KernelPlan &p, int64_t cells, int d, int L) { return bwd_plan(p, cells, d, L).bytes; }

hipError_t set_biaffine_bwd_attributes() {
    hipError_t e;
    if ((e = set_attributes<false, false>()) != hipSuccess || (e = set_attributes<false, true>()) != hipSuccess ||
        (e = set_attributes<true, false>()) != hipSuccess || (e = set_attributes<true, true>()) != hipSuccess)
        return e;
    return hipSuccess;
}

hipError_t launch_biaffine_bwd(const KernelPlan &p, int64_t cells, const void *rl, const uint8_t *rl_scales, const void *rr,
                               const uint8_t *rr_scales, const uint16_t *w, int d, int ldw, int L, const float *grad,
                               uint16_t *grad_rl, uint16_t *grad_rr, float *grad_w, char *ws, hipStream_t stream) {
    const BwdPlan b = bwd_plan(p, cells, d, L);
    const bool q8 = rl_scales != nullptr;
    uint16_t *wf = reinterpret_cast<uint16_t *>(ws + b.w_at);
    hipError_t e;
    const float *g = grad;
    const int last = p.B * p.n1 - (d < 8 ? 2 : 1);
    const Rows rl_rows{rl, rl_scales, last}, rr_rows{rr, rr_scales, last};
    // (post_cells: the square array's cells, then the compact one's)
    const int64_t *cell_at = p.post_cells + (L > 1 ? (int64_t)p.n_posts * kBlk : 0);
    if (L > 1) {
        float *gt = reinterpret_cast<float *>(ws + b.g_at);
        hipLaunchKernelGGL(bwd_compact_kernel, dim3(p.n_posts * (kBlk / 4), (L + 63) / 64), dim3(256), 0, stream, p.posts,
                           cell_at, p.post_cells, L, cells, grad, gt);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        g = gt;
    }
    if (grad_rl != nullptr || grad_rr != nullptr) {
        const int64_t pieces = (int64_t)L * 2 * b.dp * b.dp / 8;
        hipLaunchKernelGGL(bwd_weights_kernel, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, stream, w, d, ldw, b.dp,
                           pieces, wf);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        const int side0 = grad_rl != nullptr ? 0 : 1, sides = (grad_rl != nullptr) + (grad_rr != nullptr);
        float *part = b.groups > 1 ? reinterpret_cast<float *>(ws + b.part_at) : nullptr;
        BwdArgs a{};
        a.posts = p.posts;
        a.post_cells = cell_at;
        a.n_posts = p.n_posts;
        a.d = d;
        a.L = L;
        a.per_group = b.per_group;
        a.rl = rl_rows;
        a.rr = rr_rows;
        a.wf = wf;
        a.g = g;
        a.cells = cells;
        a.out[0] = grad_rl;
        a.out[1] = grad_rr;
        a.part = part;
        a.side0 = side0;
        const int n_long = p.n_long_posts;
        e = q8 ? (L > 1 ? launch_rows<true, true>(b, a, n_long, sides, stream) : launch_rows<true, false>(b, a, n_long, sides, stream))
               : (L > 1 ? launch_rows<false, true>(b, a, n_long, sides, stream) : launch_rows<false, false>(b, a, n_long, sides, stream));
        if (e != hipSuccess) return e;
        if (part != nullptr) {
            const int64_t n = (int64_t)p.n_posts * kBlk * (d / 4);
            hipLaunchKernelGGL(bwd_join_rows_kernel, dim3((unsigned)((n + 255) / 256), sides), dim3(256), 0, stream, p.posts,
                               p.n_posts, d, b.dp, b.groups, part, grad_rl, grad_rr, side0);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    if (grad_w != nullptr) {
        float *part = reinterpret_cast<float *>(ws + b.wpart_at);
        const WeightArgs a{p.posts, cell_at, p.n_posts, d, ldw, L, b.splits, b.tiles_a, b.tiles, rl_rows, rr_rows, g, cells,
                           b.splits > 1 ? part : grad_w};
        e = q8 ? (L > 1 ? launch_weight<true, true>(b, a, stream) : launch_weight<true, false>(b, a, stream))
               : (L > 1 ? launch_weight<false, true>(b, a, stream) : launch_weight<false, false>(b, a, stream));
        if (e != hipSuccess) return e;
        if (b.splits > 1) {
            const int64_t n = (int64_t)L * d * (d / 4 + 1);
            hipLaunchKernelGGL(bwd_join_weight_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, d, ldw,
                               (int64_t)L * d, b.splits, part, grad_w);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace crf
