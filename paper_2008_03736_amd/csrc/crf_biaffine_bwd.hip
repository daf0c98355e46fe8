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
// is small beside the three dense products.
//
// Roundings.  R and W are bf16, products and sums fp32.  G, which is fp32, goes
// in as bf16 hi + lo parts (at most 2^-16 of it is lost), and so does U into
// dW, which comes out in fp32.  dR^l and dR^r come out in bf16, and there U and
// X are rounded to bf16 once: each of the d terms of an output is off by at
// most 2^-8 of itself, independently, as much as the output's own rounding
// takes.
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

constexpr int kThreads = 512;                // 8 wavefronts, two per SIMD
constexpr int kBlk = kBiaRows;               // fence posts of a block
constexpr int kGS = kBlk + 8;                // row stride of the staged G (16-byte reads free of conflicts)
constexpr int kPadCols = 8;                  // padding of a staged row of R, U or X

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
// `stride`: wavefront w takes rows 8 w .. 8 w + 7, whose ids are then scalars,
// kAtOnce of them side by side, a lane eight entries of each.
template <int COLS, bool Q8>
struct Staged {
    static constexpr int kPieces = COLS / 8;                                  // of a row
    static constexpr int kAtOnce = kPieces <= 32 ? 64 / kPieces : 1;          // rows
    static constexpr int kEach = 8 / kAtOnce;
    uint4 v[kEach];   // (Q8: codes in x and y, the scale in z)
    int id[8];
    static __device__ __forceinline__ int row(int u) {   // within the wavefront's eight
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
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), k = k0 + col();
#pragma unroll
        for (int u = 0; u < 8; ++u) id[u] = constant(post + 8 * w + u);
        if constexpr (Q8) {
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
    // ONE: entry d is 1
    template <bool ONE>
    __device__ __forceinline__ void store(const Rows &r, int k0, int d, uint16_t *to, int stride) const {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), k = k0 + col();
        const bool full = k + 8 <= d, half = k + 4 == d;
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const bool row_in = id_of(u) >= 0;
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
            *reinterpret_cast<uint4 *>(to + (8 * w + row(u)) * stride + col()) = p;
        }
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
// Wavefront w takes rows 8 w .. 8 w + 7, a lane a column, so that rows are read
// along memory, what a row needs is scalar and a lane's eight rows are one
// 16-byte store of G^T[j][i]; as bf16 hi and lo parts.
struct Staged_grad {
    float v[8];
    uint32_t in;
    __device__ __forceinline__ void load(const Grad &g, const int32_t *posts, int bi, int bj) {
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int32_t *rest = posts + (size_t)bi * kPostRec + kBlk + 8 * w;
        const int64_t *cell = g.cells + (size_t)bi * kBlk + 8 * w;
        int n[8];
        int64_t c[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) n[u] = constant(rest + u);
#pragma unroll
        for (int u = 0; u < 8; ++u) c[u] = constant(cell + u);
        const int at = kBlk * (bj - bi) + lane - 8 * w;   // j - i of row 8 w
        in = 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const bool ok = at - u > 0 && at - u <= n[u];
            in |= ok ? 1u << u : 0u;
            v[u] = (g.g + c[u])[ok ? at - u : 1];   // (cell (i, i+1), which exists)
        }
    }
    __device__ __forceinline__ void store(uint16_t *hi, uint16_t *lo) const {
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        bf16x8 h, l;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float x = in >> u & 1u ? v[u] : 0.f;
            h[u] = (__bf16)x;
            l[u] = (__bf16)(x - (float)h[u]);
        }
        *reinterpret_cast<uint4 *>(hi + lane * kGS + 8 * w) = __builtin_bit_cast(uint4, h);
        *reinterpret_cast<uint4 *>(lo + lane * kGS + 8 * w) = __builtin_bit_cast(uint4, l);
    }
};
// Operands of the staged G^T, posts 16 r .. +15 by K offsets 32 ks .. +31: rows
// j with K over i, or (ROWS_I) rows i with K over j.
template <bool ROWS_I>
__device__ __forceinline__ bf16x8 grad_frag(const uint16_t *gt, int r, int ks, int lr, int lg) {
    if constexpr (ROWS_I) {
        const uint16_t *p = gt + (32 * ks + 8 * lg + (lr >> 2)) * kGS + 16 * r + 4 * (lr & 3);
        return frag_rows(p, p + 4 * kGS);
    } else {
        return frag(gt + (16 * r + lr) * kGS + 32 * ks + 8 * lg);
    }
}
// Whether that part of a block's product with itself can be other than zero
// (i < j).
template <bool ROWS_I>
__device__ __forceinline__ constexpr bool grad_part(int r, int ks) {
    return ROWS_I ? 32 * ks + 31 > 16 * r : 32 * ks < 16 * r + 15;
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
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = side ? col : k + e, a = side ? k + e : col;
        v[e] = c < d && a <= d ? wl[(size_t)c * ldw + a] : (uint16_t)0;
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
    const float *src = g + square_cells[row] * L + l0;
    const int64_t at = post_cells[row];
    for (int j0 = 1; j0 <= n; j0 += kTrCells) {
        const int m = min(kTrCells, n + 1 - j0);
        for (int c = 0; c < m; ++c)
            if (l0 + lane < L) tile[wave][c][lane] = src[(int64_t)(j0 + c) * L + lane];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        for (int t = lane; t < 64 * kTrCells; t += 64) {
            const int c = t % kTrCells, l = t / kTrCells;
            if (c < m && l0 + l < L) out[(int64_t)(l0 + l) * cells + at + j0 + c] = tile[wave][c][l];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

struct BwdArgs {
    const int32_t *posts;
    const int64_t *post_cells;
    int n_posts, d, L, per_group;   // per_group: labels of a group
    Rows rl, rr;
    const uint16_t *wf;                 // bwd_weights_kernel's fragments
    const float *g;
    int64_t cells;                      // floats between the labels of a compact gradient
    uint16_t *out[2];                   // dR^l, dR^r
    float *part;                        // [label groups][2][posts][DP]: partial sums, or NULL
    int zs;                             // items that share blocks' output columns
    int items, side0;                   // items of a side; the first grid.y's side
};

// dR^l (side 0) and dR^r (side 1) of H blocks of posts: for each label, the
// blocks' U (or X) into LDS as bf16, 64 H x DP, then its product with W's
// fragments, which come straight from L2 in the order of the lanes, each read
// by the one row of wavefronts that needs its columns.  NB: 16-column blocks
// of U per wavefront (DP = 128 NB); CB: output column blocks of a wavefront,
// WR: rows of wavefronts.
//
// A workgroup goes through items (blocks, label group, column share) on its
// own, and what the next step of staging needs (the rows of R and the cells of
// G of one pair of blocks) is in flight in registers during this step's
// products: with a workgroup an item and loads where they are needed, 5,000
// sentences at d = 500 took 418 us, 200 of them waiting for R and G.
template <int NB, int H>
struct RowsShape {
    static constexpr int kDP = 128 * NB, kPS = kDP + kPadCols;
    // U beside R, or R where U will be (U's columns are in registers until
    // every wavefront has read R)
    static constexpr bool kApart = NB <= 2;
    static constexpr int kLds = 2 * ((kApart ? 2 : 1) * H * kBlk * kPS + 2 * kBlk * kGS);
};

template <int NB, int H, int CB, int WR, bool Q8, bool COMPACT, int SIDE>
__device__ __forceinline__ void bwd_rows(const BwdArgs &a, char *smem) {
    typedef RowsShape<NB, H> S;
    constexpr int DP = S::kDP, PS = S::kPS, WC = 8 / WR, RB = 4 * H / WR;
    constexpr bool ONE = SIDE == 1, ROWS_I = SIDE == 0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 15, lg = lane >> 4;
    uint16_t *P = reinterpret_cast<uint16_t *>(smem);                  // [64 H][PS]: U or X
    uint16_t *R = S::kApart ? P + H * kBlk * PS : P;                   // [64 H][PS]: the partners' rows
    uint16_t *Gh = R + H * kBlk * PS, *Gl = Gh + kBlk * kGS;
    const int units = a.n_posts / H;
    const int wr = wave / WC, wc = wave % WC;
    const int ksteps = (a.d + 32) / 32;   // K of the dense product: d + 1 at most
    const Rows rows = SIDE == 0 ? a.rr : a.rl;

    // An item: its blocks, labels and column share.
    struct Item {
        int unit, l0, l1, cz, grp;
    };
    auto item_of = [&](int it) {
        Item x;
        x.unit = it % units;
        const int q = it / units;
        x.cz = q % a.zs;
        x.grp = q / a.zs;
        x.l0 = x.grp * a.per_group;
        x.l1 = min(x.l0 + a.per_group, a.L);
        return x;
    };
    // A block's partners: side 0 itself and those after it, side 1 those before it and itself.
    auto first_of = [&](int blk) { return SIDE == 0 ? blk : constant(a.posts + (size_t)blk * kPostRec + 2 * kBlk); };
    auto last_of = [&](int blk) { return SIDE == 0 ? constant(a.posts + (size_t)blk * kPostRec + 2 * kBlk + 1) : blk; };
    auto grad_of = [&](int l) { return Grad{a.g + (COMPACT ? l * a.cells : 0), a.post_cells}; };

    Staged<DP, Q8> sr;
    Staged_grad sg;
    auto load_step = [&](int l, int blk, int q, bool with_r) {
        sg.load(grad_of(l), a.posts, SIDE == 0 ? blk : q, SIDE == 0 ? q : blk);
        if (with_r) sr.load(rows, a.posts + (size_t)q * kPostRec, 0, a.d);
    };
    // R stays in LDS from one label to the next where blocks have one partner
    auto keeps_r = [&](int blk) { return S::kApart && first_of(blk) == last_of(blk); };

    int it = blockIdx.x;
    if (it >= a.items) return;
    Item x = item_of(it);
    load_step(x.l0, H * x.unit, first_of(H * x.unit), true);
    for (;;) {
        const int next_it = it + gridDim.x;
        const Item nx = item_of(min(next_it, a.items - 1));
        f32x4 acc[CB][RB];
        for (int l = x.l0;;) {   // (one label, l = 0, unless COMPACT)
#pragma unroll 1
            for (int h = 0; h < H; ++h) {
                const int blk = H * x.unit + h, q1 = last_of(blk);
                f32x4 u[NB][4];
#pragma unroll
                for (int c = 0; c < NB; ++c)
#pragma unroll
                    for (int r = 0; r < 4; ++r) u[c][r] = f32x4{0.f, 0.f, 0.f, 0.f};
                uint16_t *Rh = R + h * kBlk * PS;
                for (int q = first_of(blk); q <= q1; ++q) {
                    __syncthreads();   // the readers of what is stored next are done
                    if (!(l > x.l0 && keeps_r(blk))) sr.template store<ONE>(rows, 0, a.d, Rh, PS);
                    sg.store(Gh, Gl);
                    // the next step: the next partner, block, label or item
                    if (q < q1) load_step(l, blk, q + 1, true);
                    else if (h + 1 < H) load_step(l, blk + 1, first_of(blk + 1), !(l > x.l0 && keeps_r(blk + 1)));
                    else if (COMPACT && l + 1 < x.l1) load_step(l + 1, H * x.unit, first_of(H * x.unit), !keeps_r(H * x.unit));
                    else if (next_it < a.items) load_step(nx.l0, H * nx.unit, first_of(H * nx.unit), true);
                    __syncthreads();
#pragma unroll
                    for (int ks = 0; ks < 2; ++ks) {
                        bf16x8 gh[4], gl[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            gh[r] = grad_frag<ROWS_I>(Gh, r, ks, lr, lg);
                            gl[r] = grad_frag<ROWS_I>(Gl, r, ks, lr, lg);
                        }
#pragma unroll
                        for (int c = 0; c < NB; ++c) {
                            const uint16_t *p = Rh + (32 * ks + 8 * lg + (lr >> 2)) * PS + 16 * (wave * NB + c) + 4 * (lr & 3);
                            const bf16x8 rf = frag_rows(p, p + 4 * PS);
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (grad_part<ROWS_I>(r, ks) || q != blk) {
                                    u[c][r] = mfma(rf, gh[r], u[c][r]);
                                    u[c][r] = mfma(rf, gl[r], u[c][r]);
                                }
                        }
                    }
                }
                if constexpr (!S::kApart) __syncthreads();   // R's readers are done
                // u[c][r]: columns 16 (wave NB + c) + 4 lg .. +3 of post 16 r + lr
#pragma unroll
                for (int c = 0; c < NB; ++c)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        *reinterpret_cast<bf16x4 *>(P + (h * kBlk + 16 * r + lr) * PS + 16 * (wave * NB + c) + 4 * lg) =
                            __builtin_convertvector(u[c][r], bf16x4);
            }
            __syncthreads();

            if (!COMPACT || l == x.l0)
#pragma unroll
                for (int c = 0; c < CB; ++c)
#pragma unroll
                    for (int r = 0; r < RB; ++r) acc[c][r] = f32x4{0.f, 0.f, 0.f, 0.f};
            const int col0 = (x.cz * WC + wc) * CB;   // the wavefront's first output column block
            const uint16_t *wf = a.wf + ((((size_t)l * 2 + SIDE) * (DP / 32)) * (DP / 16) + col0) * 512 + 8 * lane;
            const uint16_t *prow = P + (wr * RB * 16 + lr) * PS + 8 * lg;
            bf16x8 wv[2][CB];   // two steps of W
#pragma unroll
            for (int c = 0; c < CB; ++c) wv[0][c] = frag(wf + (size_t)c * 512);
            auto dense_step = [&](int ks, bf16x8 (&now)[CB], bf16x8 (&then)[CB]) {
                const int kn = min(ks + 1, ksteps - 1);
#pragma unroll
                for (int c = 0; c < CB; ++c) then[c] = frag(wf + ((size_t)kn * (DP / 16) + c) * 512);
                bf16x8 pv = frag(prow + 32 * ks);
                __builtin_amdgcn_sched_barrier(0);   // (left alone, they are issued where they are waited for)
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    bf16x8 pn = pv;
                    if (r + 1 < RB) pn = frag(prow + 16 * (r + 1) * PS + 32 * ks);
#pragma unroll
                    for (int c = 0; c < CB; ++c) acc[c][r] = mfma(now[c], pv, acc[c][r]);
                    pv = pn;
                }
                __builtin_amdgcn_sched_barrier(0);
            };
            int ks = 0;
            for (; ks + 1 < ksteps; ks += 2) {
                dense_step(ks, wv[0], wv[1]);
                dense_step(ks + 1, wv[1], wv[0]);
            }
            if (ks < ksteps) dense_step(ks, wv[0], wv[1]);
            if (!COMPACT || ++l >= x.l1) break;
        }

        // acc[c][r]: columns 16 (col0 + c) + 4 lg .. +3 of post 16 (wr RB + r) + lr
        const int col0 = (x.cz * WC + wc) * CB;
        int ids[RB];   // (all before the first store, which a later load would wait for)
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int slot = 16 * (wr * RB + r) + lr;
            ids[r] = a.posts[(size_t)(H * x.unit + slot / kBlk) * kPostRec + slot % kBlk];
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int slot = 16 * (wr * RB + r) + lr, id = ids[r];
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                const int col = 16 * (col0 + c) + 4 * lg;
                if (id < 0 || col >= a.d) continue;
                if (a.part != nullptr)
                    *reinterpret_cast<f32x4 *>(a.part + (((size_t)x.grp * 2 + SIDE) * a.n_posts * kBlk + H * kBlk * x.unit + slot) * DP + col) =
                        acc[c][r];
                else
                    *reinterpret_cast<bf16x4 *>(a.out[SIDE] + (size_t)id * a.d + col) = __builtin_convertvector(acc[c][r], bf16x4);
            }
        }
        if (next_it >= a.items) break;
        it = next_it;
        x = nx;
    }
}

template <int NB, int H, int CB, int WR, bool Q8, bool COMPACT>
__global__ __launch_bounds__(kThreads) void bwd_rows_kernel(BwdArgs a) {
    extern __shared__ __align__(16) char smem[];
    if (blockIdx.y + a.side0 == 0) bwd_rows<NB, H, CB, WR, Q8, COMPACT, 0>(a, smem);
    else bwd_rows<NB, H, CB, WR, Q8, COMPACT, 1>(a, smem);
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
    for (int q = 0; q < groups; ++q)
        s += *reinterpret_cast<const f32x4 *>(part + (((size_t)q * 2 + side) * n_posts * kBlk + slot) * dp + col);
    *reinterpret_cast<bf16x4 *>((side ? out_r : out_l) + (size_t)id * d + col) = __builtin_convertvector(s, bf16x4);
}

// dW of one label, a tile of 128 T columns a by 128 T rows c, over a share of
// the blocks of posts: a wavefront holds U of its 16 T columns c in registers,
// whose layout is that of the second product's operand when K is numbered so
// that a lane's eight posts are 4 lg .. +3 of two 16-post blocks.
struct WeightArgs {
    const int32_t *posts;
    const int64_t *post_cells;
    int n_posts, d, ldw, splits, tiles_a;
    Rows rl, rr;
    const float *g;
    int64_t cells;
    float *out;   // splits = 1: dW [L][d][ldw]; else partial sums [splits][L][d][d + 4]
};
template <int T>
struct WeightShape {
    static constexpr int kT = 128 * T, kTS = kT + kPadCols;
    static constexpr int kLds = 2 * (2 * kBlk * kTS + 2 * kBlk * kGS);
};

template <int T, bool Q8, bool COMPACT>
__global__ __launch_bounds__(kThreads) void bwd_weight_kernel(WeightArgs a) {
    extern __shared__ __align__(16) char smem[];
    typedef WeightShape<T> S;
    constexpr int TS = S::kTS, AB = 8 * T;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 15, lg = lane >> 4;
    uint16_t *Ra = reinterpret_cast<uint16_t *>(smem), *Rc = Ra + kBlk * TS, *Gh = Rc + kBlk * TS, *Gl = Gh + kBlk * kGS;
    const int a0 = S::kT * ((int)blockIdx.x % a.tiles_a), c0 = S::kT * ((int)blockIdx.x / a.tiles_a);
    const int l = blockIdx.y, split = blockIdx.z;
    const int b0 = (int)((int64_t)a.n_posts * split / a.splits), b1 = (int)((int64_t)a.n_posts * (split + 1) / a.splits);
    const Grad g{a.g + (COMPACT ? l * a.cells : 0), a.post_cells};

    f32x4 acc[AB][T];
#pragma unroll
    for (int x = 0; x < AB; ++x)
#pragma unroll
        for (int c = 0; c < T; ++c) acc[x][c] = f32x4{0.f, 0.f, 0.f, 0.f};

    Staged<S::kT, Q8> sa, sc;
    Staged_grad sg;
    auto load_step = [&](int blk, int q) {
        sg.load(g, a.posts, blk, q);
        sc.load(a.rr, a.posts + (size_t)q * kPostRec, c0, a.d);
        if (q == blk) sa.load(a.rl, a.posts + (size_t)blk * kPostRec, a0, a.d);
    };
    if (b0 < b1) load_step(b0, b0);
    for (int blk = b0; blk < b1; ++blk) {
        const int last = constant(a.posts + (size_t)blk * kPostRec + 2 * kBlk + 1);
        f32x4 u[4][T];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < T; ++c) u[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int q = blk; q <= last; ++q) {
            __syncthreads();
            if (q == blk) sa.template store<true>(a.rl, a0, a.d, Ra, TS);
            sc.template store<false>(a.rr, c0, a.d, Rc, TS);
            sg.store(Gh, Gl);
            if (q < last) load_step(blk, q + 1);
            else if (blk + 1 < b1) load_step(blk + 1, blk + 1);
            __syncthreads();
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int c = 0; c < T; ++c) {
                    const uint16_t *p = Rc + (32 * ks + 8 * lg + (lr >> 2)) * TS + 16 * (wave * T + c) + 4 * (lr & 3);
                    const bf16x8 rf = frag_rows(p, p + 4 * TS);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (grad_part<true>(r, ks) || q != blk) {
                            u[r][c] = mfma(grad_frag<true>(Gh, r, ks, lr, lg), rf, u[r][c]);
                            u[r][c] = mfma(grad_frag<true>(Gl, r, ks, lr, lg), rf, u[r][c]);
                        }
                }
        }
#pragma unroll
        for (int kp = 0; kp < 2; ++kp) {
            bf16x8 hi[T], lo[T];
#pragma unroll
            for (int c = 0; c < T; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const float v = u[2 * kp + e][c][t];
                        const __bf16 h = (__bf16)v;
                        hi[c][4 * e + t] = h;
                        lo[c][4 * e + t] = (__bf16)(v - (float)h);
                    }
            const uint16_t *p = Ra + (32 * kp + 4 * lg + (lr >> 2)) * TS + 4 * (lr & 3);
#pragma unroll
            for (int x = 0; x < AB; ++x) {
                const bf16x8 rf = frag_rows(p + 16 * x, p + 16 * TS + 16 * x);
#pragma unroll
                for (int c = 0; c < T; ++c) {
                    acc[x][c] = mfma(rf, hi[c], acc[x][c]);
                    acc[x][c] = mfma(rf, lo[c], acc[x][c]);
                }
            }
        }
    }

    // acc[x][c]: a = a0 + 16 x + 4 lg .. +3 of row c0 + 16 (wave T + c) + lr
    const bool whole = a.splits == 1;
    const int stride = whole ? a.ldw : a.d + 4;
    float *out = a.out + ((size_t)split * gridDim.y + l) * a.d * stride;
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
    for (int q = 0; q < splits; ++q) s += *reinterpret_cast<const f32x4 *>(p + (size_t)q * rows * (d + 4));
    float *at = out + row * ldw + col;
    if (col < d) *reinterpret_cast<f32x4 *>(at) = s;
    else *at = s[0];
}

// ---------------------------------------------------------------------------
// Launches.

inline int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

constexpr int kCus = 256;

// How a call is cut up, and its workspace.
struct BwdPlan {
    int nb, dp;                     // DP = 128 nb
    bool small;                     // few blocks: a block an item, its columns shared by nb items
    int h, zs, groups, per_group;   // blocks of an item; column shares; label groups and labels of one
    int t, tiles_a, tiles_c, splits;
    int64_t w_at, g_at, part_at, wpart_at, bytes;
};
BwdPlan bwd_plan(const KernelPlan &p, int64_t cells, int d, int L) {
    BwdPlan b{};
    b.nb = (d + 1 + 127) / 128;
    b.dp = 128 * b.nb;
    b.small = (int64_t)p.n_posts * L < 256;
    b.h = b.small || b.nb == 1 ? 1 : 2;
    b.zs = b.small ? b.nb : 1;
    const int64_t items = (int64_t)p.n_posts / b.h * 2;
    b.groups = (int)std::max<int64_t>(1, std::min<int64_t>(L, 2 * kCus / items));
    b.per_group = (L + b.groups - 1) / b.groups;
    b.groups = (L + b.per_group - 1) / b.per_group;
    b.t = d + 1 > 128 ? 2 : 1;
    b.tiles_a = (d + 1 + 128 * b.t - 1) / (128 * b.t);
    b.tiles_c = (d + 128 * b.t - 1) / (128 * b.t);
    const int64_t wgs = (int64_t)b.tiles_a * b.tiles_c * L;
    b.splits = (int)std::max<int64_t>(1, std::min<int64_t>(p.n_posts, (b.t == 2 ? kCus : 3 * kCus) / wgs));
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

template <int NB, int H, int CB, int WR, bool Q8, bool COMPACT>
hipError_t launch_rows(const BwdArgs &a, int sides, int per_cu, hipStream_t stream) {
    const int slots = std::max(1, per_cu * kCus / sides);
    hipLaunchKernelGGL((bwd_rows_kernel<NB, H, CB, WR, Q8, COMPACT>), dim3(std::min(a.items, slots), sides), dim3(kThreads),
                       (RowsShape<NB, H>::kLds), stream, a);
    return hipGetLastError();
}
// Every build of bwd_rows_kernel, with the workgroups of one that a CU holds.
#define CRF_BWD_ROWS(F)                                                                             \
    F(1, false, 1, 1, 2, 2, 2) F(2, false, 2, 2, 4, 2, 1) F(3, false, 3, 2, 3, 1, 1) F(4, false, 4, 2, 4, 1, 1) \
    F(1, true, 1, 1, 1, 1, 2) F(2, true, 2, 1, 1, 1, 1) F(3, true, 3, 1, 1, 1, 1) F(4, true, 4, 1, 1, 1, 1)
template <bool Q8, bool COMPACT>
hipError_t launch_rows_of(const BwdPlan &b, const BwdArgs &a, int sides, hipStream_t stream) {
#define CRF_LAUNCH(N, SMALL, NB, H, CB, WR, PER) \
    if (b.nb == N && b.small == SMALL) return launch_rows<NB, H, CB, WR, Q8, COMPACT>(a, sides, PER, stream);
    CRF_BWD_ROWS(CRF_LAUNCH)
#undef CRF_LAUNCH
    return hipErrorInvalidValue;
}
template <bool Q8, bool COMPACT>
hipError_t launch_weight(const BwdPlan &b, const WeightArgs &a, int L, hipStream_t stream) {
    const dim3 grid(b.tiles_a * b.tiles_c, L, b.splits);
    if (b.t == 1)
        hipLaunchKernelGGL((bwd_weight_kernel<1, Q8, COMPACT>), grid, dim3(kThreads), WeightShape<1>::kLds, stream, a);
    else
        hipLaunchKernelGGL((bwd_weight_kernel<2, Q8, COMPACT>), grid, dim3(kThreads), WeightShape<2>::kLds, stream, a);
    return hipGetLastError();
}

template <bool Q8, bool COMPACT>
hipError_t set_attributes() {
    hipError_t e;
    auto set = [&](const void *f, int bytes) { return hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); };
#define CRF_SET(N, SMALL, NB, H, CB, WR, PER) \
    if ((e = set((const void *)bwd_rows_kernel<NB, H, CB, WR, Q8, COMPACT>, RowsShape<NB, H>::kLds)) != hipSuccess) return e;
    CRF_BWD_ROWS(CRF_SET)
#undef CRF_SET
    if ((e = set((const void *)bwd_weight_kernel<1, Q8, COMPACT>, WeightShape<1>::kLds)) != hipSuccess ||
        (e = set((const void *)bwd_weight_kernel<2, Q8, COMPACT>, WeightShape<2>::kLds)) != hipSuccess)
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
        const BwdArgs a{p.posts, cell_at, p.n_posts, d, L, b.per_group, rl_rows, rr_rows,
                        wf, g, cells, {grad_rl, grad_rr}, part, b.zs, p.n_posts / b.h * b.zs * b.groups, side0};
        e = q8 ? (L > 1 ? launch_rows_of<true, true>(b, a, sides, stream) : launch_rows_of<true, false>(b, a, sides, stream))
               : (L > 1 ? launch_rows_of<false, true>(b, a, sides, stream) : launch_rows_of<false, false>(b, a, sides, stream));
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
        const WeightArgs a{p.posts, cell_at, p.n_posts, d, ldw, b.splits, b.tiles_a, rl_rows, rr_rows, g, cells, b.splits > 1 ? part : grad_w};
        e = q8 ? (L > 1 ? launch_weight<true, true>(b, a, L, stream) : launch_weight<true, false>(b, a, L, stream))
               : (L > 1 ? launch_weight<false, true>(b, a, L, stream) : launch_weight<false, false>(b, a, L, stream));
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
