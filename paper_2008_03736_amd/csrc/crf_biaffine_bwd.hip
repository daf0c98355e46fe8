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
};
// Entries k .. k+7 of row `id` (k a multiple of 8, d one of 4), zero past d;
// ONE: entry d is 1.
template <bool Q8, bool ONE>
__device__ __forceinline__ uint4 load_piece(const Rows &r, int id, int k, int d) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (id >= 0 && k < d) {
        if constexpr (Q8) {
            const int wide = row_codes(d);
            v = eight_of_codes(*reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(r.x) + (size_t)id * wide + k),
                               r.scales[(size_t)id * (wide / kRowBlock) + k / kRowBlock]);
            if (k + 4 >= d) v.z = v.w = 0u;
        } else {
            const uint16_t *row = static_cast<const uint16_t *>(r.x) + (size_t)id * d + k;
            const uint2 a = *reinterpret_cast<const uint2 *>(row);
            v.x = a.x;
            v.y = a.y;
            if (k + 4 < d) {
                const uint2 b = *reinterpret_cast<const uint2 *>(row + 4);
                v.z = b.x;
                v.w = b.y;
            }
        }
    }
    if constexpr (ONE) {
        if (id >= 0 && k == d) v.x = 0x3F80u;
        if (id >= 0 && k + 4 == d) v.z = 0x3F80u;
    }
    return v;
}

// Columns k0 .. k0 + COLS of a block's rows into LDS (row stride `stride`).
template <bool Q8, bool ONE, int COLS>
__device__ __forceinline__ void stage_rows(const Rows &r, const int32_t *ids, int k0, int d, uint16_t *to, int stride) {
    constexpr int kPieces = COLS / 8, kEach = kBlk * kPieces / kThreads;
    uint4 v[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int t = (int)threadIdx.x + kThreads * u;
        v[u] = load_piece<Q8, ONE>(r, ids[t / kPieces], k0 + 8 * (t % kPieces), d);
    }
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int t = (int)threadIdx.x + kThreads * u;
        *reinterpret_cast<uint4 *>(to + t / kPieces * stride + 8 * (t % kPieces)) = v[u];
    }
}

// Where a label's gradient lies: the caller's [B][N1][N1] (COMPACT false), or
// the compact cells of the label.
struct Grad {
    const float *g;
    const int64_t *cells;   // KernelPlan::post_cells
    int N1;
};
// G of rows i in block `bi` and columns j in block `bj` as bf16 hi and lo
// parts, [i][j], or [j][i] where TR: the cells of one sentence with i < j,
// zero elsewhere (other cells are not read).
template <bool COMPACT, bool TR>
__device__ __forceinline__ void stage_grad(const Grad &g, const int32_t *posts, int bi, int bj, uint16_t *hi, uint16_t *lo) {
    constexpr int kEach = kBlk / (kThreads / 64);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t *ri = posts + (size_t)bi * kPostRec, *rj = posts + (size_t)bj * kPostRec;
    const int idj = rj[lane], basej = rj[kBlk + lane];
    float v[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int r = wave + (kThreads / 64) * u, idi = ri[r];
        const bool in = idi >= 0 && idj > idi && ri[kBlk + r] == basej;
        v[u] = 0.f;
        if (in) v[u] = g.g[(COMPACT ? g.cells[(size_t)bi * kBlk + r] : (int64_t)idi * g.N1) + (idj - basej)];
    }
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int r = wave + (kThreads / 64) * u, at = TR ? lane * kGS + r : r * kGS + lane;
        const __bf16 h = (__bf16)v[u];
        hi[at] = __builtin_bit_cast(uint16_t, h);
        lo[at] = __builtin_bit_cast(uint16_t, (__bf16)(v[u] - (float)h));
    }
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
                                                          const int32_t *__restrict__ len, int N1, int L, int64_t cells,
                                                          const float *__restrict__ g, float *__restrict__ out) {
    __shared__ float tile[4][kTrCells][65];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = (int)blockIdx.x * 4 + wave, l0 = (int)blockIdx.y * 64;
    const int32_t *rec = posts + (size_t)(row / kBlk) * kPostRec + row % kBlk;
    const int id = rec[0];
    if (id < 0) return;   // (wavefronts share nothing)
    const int base = rec[kBlk], i = id - base, n = len[base / N1];
    const float *src = g + ((int64_t)id * N1) * L + l0;
    const int64_t at = post_cells[row];
    for (int j0 = i + 1; j0 <= n; j0 += kTrCells) {
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
    int n_posts, N1, d, L, per_group;   // per_group: labels of a workgroup
    Rows rl, rr;
    const uint16_t *wf;                 // bwd_weights_kernel's fragments
    const float *g;
    int64_t cells;                      // floats between the labels of a compact gradient
    uint16_t *out[2];                   // dR^l, dR^r
    float *part;                        // [label groups][2][posts][16 * column blocks]: partial sums, or NULL
    int zs;                             // workgroups that share a pair of blocks' output columns
    int side0;                          // the first grid.y's side
};

// dR^l (side 0) and dR^r (side 1) of two blocks of posts: for each label, the
// blocks' U (or X) into LDS as bf16, 128 x DP, then its product with W's
// fragments, which come straight from L2 in the order of the lanes, each read
// by the one row of wavefronts that needs its columns.  NB: 16-column blocks
// of U per wavefront (DP = 128 NB); CB: output column blocks of a wavefront,
// WR: rows of wavefronts.
template <int NB>
struct RowsShape {
    static constexpr int kDP = 128 * NB, kPS = kDP + kPadCols;
    // U of 128 posts beside R, or R where U will be (its columns are in
    // registers until every wavefront has read R)
    static constexpr bool kApart = NB <= 2;
    static constexpr int kLds = 2 * ((kApart ? 4 : 2) * kBlk * kPS + 2 * kBlk * kGS);
};

template <int NB, int CB, int WR, bool Q8, bool COMPACT, int SIDE>
__device__ __forceinline__ void bwd_rows(const BwdArgs &a, char *smem) {
    typedef RowsShape<NB> S;
    constexpr int DP = S::kDP, PS = S::kPS, WC = 8 / WR, RB = 8 / WR;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 15, lg = lane >> 4;
    uint16_t *P = reinterpret_cast<uint16_t *>(smem);                  // [128][PS]: U or X
    uint16_t *R = S::kApart ? P + 2 * kBlk * PS : P;                   // [128][PS]: the partners' rows
    uint16_t *Gh = R + 2 * kBlk * PS, *Gl = Gh + kBlk * kGS;
    const int pair = blockIdx.x, cz = (int)blockIdx.z % a.zs, grp = (int)blockIdx.z / a.zs;
    const int l0 = grp * a.per_group, l1 = min(l0 + a.per_group, a.L);
    const int wr = wave / WC, wc = wave % WC, col0 = (cz * WC + wc) * CB;   // first output column block
    const int ksteps = (a.d + 32) / 32;                                      // K of the dense product: d + 1 at most

    f32x4 acc[CB][RB];
    for (int l = l0;;) {   // (one label, l = 0, unless COMPACT)
        const Grad g{a.g + (COMPACT ? l * a.cells : 0), a.post_cells, a.N1};
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            const int blk = 2 * pair + h;
            if (blk >= a.n_posts) break;
            const int32_t *rec = a.posts + (size_t)blk * kPostRec;
            const int first = rec[2 * kBlk], last = rec[2 * kBlk + 1];
            const int q0 = SIDE == 0 ? blk : first, q1 = SIDE == 0 ? last : blk;
            f32x4 u[NB][4];
#pragma unroll
            for (int c = 0; c < NB; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) u[c][r] = f32x4{0.f, 0.f, 0.f, 0.f};
            uint16_t *Rh = R + h * kBlk * PS;
            for (int q = q0; q <= q1; ++q) {
                __syncthreads();   // the readers of what is staged next are done
                if (!(S::kApart && l > l0 && first == last))
                    stage_rows<Q8, SIDE == 1, DP>(SIDE == 0 ? a.rr : a.rl, a.posts + (size_t)q * kPostRec, 0, a.d, Rh, PS);
                stage_grad<COMPACT, SIDE == 1>(g, a.posts, SIDE == 0 ? blk : q, SIDE == 0 ? q : blk, Gh, Gl);
                __syncthreads();
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    bf16x8 gh[4], gl[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        gh[r] = frag(Gh + (16 * r + lr) * kGS + 32 * ks + 8 * lg);
                        gl[r] = frag(Gl + (16 * r + lr) * kGS + 32 * ks + 8 * lg);
                    }
#pragma unroll
                    for (int c = 0; c < NB; ++c) {
                        const uint16_t *p = Rh + (32 * ks + 8 * lg + (lr >> 2)) * PS + 16 * (wave * NB + c) + 4 * (lr & 3);
                        const bf16x8 rf = frag_rows(p, p + 4 * PS);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
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

        if (!COMPACT || l == l0)
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int r = 0; r < RB; ++r) acc[c][r] = f32x4{0.f, 0.f, 0.f, 0.f};
        const uint16_t *wf = a.wf + ((((size_t)l * 2 + SIDE) * (DP / 32)) * (DP / 16) + col0) * 512 + 8 * lane;
        const uint16_t *prow = P + (wr * RB * 16 + lr) * PS + 8 * lg;
        for (int ks = 0; ks < ksteps; ++ks) {
            bf16x8 wv[CB];
#pragma unroll
            for (int c = 0; c < CB; ++c) wv[c] = frag(wf + ((size_t)ks * (DP / 16) + c) * 512);
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const bf16x8 pv = frag(prow + 16 * r * PS + 32 * ks);
#pragma unroll
                for (int c = 0; c < CB; ++c) acc[c][r] = mfma(wv[c], pv, acc[c][r]);
            }
        }
        if (!COMPACT || ++l >= l1) break;
    }

    // acc[c][r]: columns 16 (col0 + c) + 4 lg .. +3 of post 16 (wr RB + r) + lr
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int slot = 16 * (wr * RB + r) + lr, blk = 2 * pair + slot / kBlk;
        const int id = blk < a.n_posts ? a.posts[(size_t)blk * kPostRec + slot % kBlk] : -1;
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            const int col = 16 * (col0 + c) + 4 * lg;
            if (id < 0 || col >= a.d) continue;
            if (a.part != nullptr)
                *reinterpret_cast<f32x4 *>(a.part + (((size_t)grp * 2 + SIDE) * a.n_posts * kBlk + blk * kBlk + slot % kBlk) * DP + col) =
                    acc[c][r];
            else
                *reinterpret_cast<bf16x4 *>(a.out[SIDE] + (size_t)id * a.d + col) = __builtin_convertvector(acc[c][r], bf16x4);
        }
    }
}

template <int NB, int CB, int WR, bool Q8, bool COMPACT>
__global__ __launch_bounds__(kThreads) void bwd_rows_kernel(BwdArgs a) {
    extern __shared__ __align__(16) char smem[];
    if (blockIdx.y + a.side0 == 0) bwd_rows<NB, CB, WR, Q8, COMPACT, 0>(a, smem);
    else bwd_rows<NB, CB, WR, Q8, COMPACT, 1>(a, smem);
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
    int n_posts, N1, d, ldw, splits, tiles_a;
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
    const Grad g{a.g + (COMPACT ? l * a.cells : 0), a.post_cells, a.N1};

    f32x4 acc[AB][T];
#pragma unroll
    for (int x = 0; x < AB; ++x)
#pragma unroll
        for (int c = 0; c < T; ++c) acc[x][c] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int blk = b0; blk < b1; ++blk) {
        const int last = a.posts[(size_t)blk * kPostRec + 2 * kBlk + 1];
        f32x4 u[4][T];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < T; ++c) u[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int q = blk; q <= last; ++q) {
            __syncthreads();
            if (q == blk) stage_rows<Q8, true, S::kT>(a.rl, a.posts + (size_t)blk * kPostRec, a0, a.d, Ra, TS);
            stage_rows<Q8, false, S::kT>(a.rr, a.posts + (size_t)q * kPostRec, c0, a.d, Rc, TS);
            stage_grad<COMPACT, false>(g, a.posts, blk, q, Gh, Gl);
            __syncthreads();
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int c = 0; c < T; ++c) {
                    const uint16_t *p = Rc + (32 * ks + 8 * lg + (lr >> 2)) * TS + 16 * (wave * T + c) + 4 * (lr & 3);
                    const bf16x8 rf = frag_rows(p, p + 4 * TS);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        u[r][c] = mfma(frag(Gh + (16 * r + lr) * kGS + 32 * ks + 8 * lg), rf, u[r][c]);
                        u[r][c] = mfma(frag(Gl + (16 * r + lr) * kGS + 32 * ks + 8 * lg), rf, u[r][c]);
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

// How a call is cut up, and its workspace.
struct BwdPlan {
    int nb, dp;                     // DP = 128 nb
    int zs, groups, per_group;      // column shares; label groups and labels of one
    int t, tiles_a, tiles_c, splits;
    int64_t w_at, g_at, part_at, wpart_at, bytes;
};
BwdPlan bwd_plan(const KernelPlan &p, int64_t cells, int d, int L) {
    BwdPlan b{};
    b.nb = (d + 1 + 127) / 128;
    b.dp = 128 * b.nb;
    const int pairs = (p.n_posts + 1) / 2;
    b.zs = 1;
    b.groups = std::max(1, std::min(L, 512 / (2 * pairs)));
    b.per_group = (L + b.groups - 1) / b.groups;
    b.groups = (L + b.per_group - 1) / b.per_group;
    b.t = d + 1 > 128 ? 2 : 1;
    b.tiles_a = (d + 1 + 128 * b.t - 1) / (128 * b.t);
    b.tiles_c = (d + 128 * b.t - 1) / (128 * b.t);
    const int64_t wgs = (int64_t)b.tiles_a * b.tiles_c * L;
    b.splits = (int)std::max<int64_t>(1, std::min<int64_t>(p.n_posts, (b.t == 2 ? 256 : 768) / wgs));
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

template <int NB, int CB, int WR, bool Q8, bool COMPACT>
hipError_t launch_rows(const BwdArgs &a, int sides, int groups, hipStream_t stream) {
    hipLaunchKernelGGL((bwd_rows_kernel<NB, CB, WR, Q8, COMPACT>), dim3((a.n_posts + 1) / 2, sides, a.zs * groups),
                       dim3(kThreads), RowsShape<NB>::kLds, stream, a);
    return hipGetLastError();
}
template <bool Q8, bool COMPACT>
hipError_t launch_rows_nb(int nb, const BwdArgs &a, int sides, int groups, hipStream_t stream) {
    switch (nb) {
        case 1: return launch_rows<1, 2, 2, Q8, COMPACT>(a, sides, groups, stream);
        case 2: return launch_rows<2, 4, 2, Q8, COMPACT>(a, sides, groups, stream);
        case 3: return launch_rows<3, 3, 1, Q8, COMPACT>(a, sides, groups, stream);
        default: return launch_rows<4, 4, 1, Q8, COMPACT>(a, sides, groups, stream);
    }
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
    if ((e = set((const void *)bwd_rows_kernel<1, 2, 2, Q8, COMPACT>, RowsShape<1>::kLds)) != hipSuccess ||
        (e = set((const void *)bwd_rows_kernel<2, 4, 2, Q8, COMPACT>, RowsShape<2>::kLds)) != hipSuccess ||
        (e = set((const void *)bwd_rows_kernel<3, 3, 1, Q8, COMPACT>, RowsShape<3>::kLds)) != hipSuccess ||
        (e = set((const void *)bwd_rows_kernel<4, 4, 1, Q8, COMPACT>, RowsShape<4>::kLds)) != hipSuccess ||
        (e = set((const void *)bwd_weight_kernel<1, Q8, COMPACT>, WeightShape<1>::kLds)) != hipSuccess ||
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
    if (L > 1) {
        float *gt = reinterpret_cast<float *>(ws + b.g_at);
        hipLaunchKernelGGL(bwd_compact_kernel, dim3(p.n_posts * (kBlk / 4), (L + 63) / 64), dim3(256), 0, stream, p.posts,
                           p.post_cells, p.len, p.n1, L, cells, grad, gt);
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
        const BwdArgs a{p.posts, p.post_cells, p.n_posts, p.n1, d, L, b.per_group, Rows{rl, rl_scales}, Rows{rr, rr_scales},
                        wf, g, cells, {grad_rl, grad_rr}, part, b.zs, side0};
        e = q8 ? (L > 1 ? launch_rows_nb<true, true>(b.nb, a, sides, b.groups, stream)
                        : launch_rows_nb<true, false>(b.nb, a, sides, b.groups, stream))
               : (L > 1 ? launch_rows_nb<false, true>(b.nb, a, sides, b.groups, stream)
                        : launch_rows_nb<false, false>(b.nb, a, sides, b.groups, stream));
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
        const WeightArgs a{p.posts, p.post_cells, p.n_posts, p.n1, d, ldw, b.splits, b.tiles_a, Rows{rl, rl_scales},
                           Rows{rr, rr_scales}, g, cells, b.splits > 1 ? part : grad_w};
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
