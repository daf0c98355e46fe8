// crf_rows.hip -- activation rows in 8 bits.
//
// A row of d bf16 values is held as blocks of kRowBlock = 32 codes that share
// a power of two: with m the block's largest magnitude,
//     s = ceil(log2(m / 448)),  code = e4m3(x 2^-s),  x' = code 2^s,
// so that the largest code's magnitude lies in (224, 448], e4m3's topmost
// binade and a half, and no value overflows.  A value x is off by at most the
// larger of 2^-4 |x| and 2^-10 2^s: by 2^-4 |x| from 2^-6 2^s on, where e4m3 has
// four digits, and so within 2^-13 of its block's largest (2^-6 / 224 < 2^-13).
// The power is held as a byte, s + 127 (at least 0).
//
// Memory-bound: 2 bytes read and 1 + 1/32 written an entry, and back.  Four
// lanes take a block (16 bytes of bf16 each), so a block's largest magnitude
// is two lane exchanges, and a lane's eight codes are one 8-byte store.  The
// plan's lists of fence posts give the rows, so that padded ones cost nothing.
// 5,000 sentences at d = 500: packing 58.7 us, unpacking 39.4, 198 MB each:
// 3.4 and 5.0 TB/s (a large copy reaches 5.1).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "crf_internal.h"
#include "crf_rows.h"

namespace crf {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowsPerGroup = 16;   // rows a workgroup takes

// Eight bf16 of a row from entry k (zeros past entry d - 1; d is a multiple
// of 4 and rows are 8-byte aligned).
__device__ __forceinline__ uint4 load_eight(const uint16_t *row, int k, int d) {
    const uint2 z = make_uint2(0u, 0u);
    const uint2 x = k < d ? *reinterpret_cast<const uint2 *>(row + k) : z;
    const uint2 y = k + 4 < d ? *reinterpret_cast<const uint2 *>(row + k + 4) : z;
    return make_uint4(x.x, x.y, y.x, y.y);
}

__global__ __launch_bounds__(kRowThreads) void pack_rows_kernel(const int32_t *__restrict__ posts, int d,
                                                                const uint16_t *__restrict__ x,
                                                                uint8_t *__restrict__ codes,
                                                                uint8_t *__restrict__ scales) {
    const int wide = row_codes(d), per = wide / 8;   // lanes a row
    const int32_t *ids = posts + (size_t)(blockIdx.x / (kBiaRows / kRowsPerGroup)) * kPostRec +
                         blockIdx.x % (kBiaRows / kRowsPerGroup) * kRowsPerGroup;
    for (int t = threadIdx.x; t < kRowsPerGroup * per; t += kRowThreads) {
        const int r = t / per, k = 8 * (t - r * per), id = ids[r];
        if (id < 0) continue;   // (the four lanes of a block are of one row)
        const uint4 v = load_eight(x + (size_t)id * d, k, d);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t top = 0;   // the largest finite magnitude's bits
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t m = w[q] >> (16 * h) & 0x7FFFu;
                top = max(top, m < 0x7F80u ? m : 0u);
            }
        top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
        // m = (1 + f/128) 2^(e - 127): s = e - 127 - 8, one more past 1.75
        const int s = max((int)(top >> 7) - 8 + ((top & 127u) > 96u ? 1 : 0), 0);
        const float inv = __builtin_bit_cast(float, (uint32_t)(254 - s) << 23);   // 2^(127 - s)
        // bf16's last 1/16 of a binade would round to 2^128, which it does not
        // hold: there the code below is taken
        const float most = s == 247 ? 240.f : 448.f;
        auto scaled = [&](uint32_t bits) {
            return __builtin_amdgcn_fmed3f(__builtin_bit_cast(float, bits) * inv, -most, most);
        };
        uint32_t out[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            int c = 0;
            const uint32_t lo = w[2 * q], hi = w[2 * q + 1];
            c = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(lo << 16), scaled(lo & 0xFFFF0000u), c, false);
            c = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(hi << 16), scaled(hi & 0xFFFF0000u), c, true);
            // infinities and NaN: the code's NaN
            uint32_t bad = 0;
            bad |= (lo & 0x7F80u) == 0x7F80u ? 0x7Fu : 0u;
            bad |= (lo & 0x7F800000u) == 0x7F800000u ? 0x7F00u : 0u;
            bad |= (hi & 0x7F80u) == 0x7F80u ? 0x7F0000u : 0u;
            bad |= (hi & 0x7F800000u) == 0x7F800000u ? 0x7F000000u : 0u;
            out[q] = (uint32_t)c | bad;
        }
        *reinterpret_cast<uint2 *>(codes + (size_t)id * wide + k) = make_uint2(out[0], out[1]);
        if ((t & 3) == 0) scales[(size_t)id * (wide / kRowBlock) + k / kRowBlock] = (uint8_t)s;
    }
}

__global__ __launch_bounds__(kRowThreads) void unpack_rows_kernel(const int32_t *__restrict__ posts, int d,
                                                                  const uint8_t *__restrict__ codes,
                                                                  const uint8_t *__restrict__ scales,
                                                                  uint16_t *__restrict__ x) {
    const int wide = row_codes(d), per = wide / 8;
    const int32_t *ids = posts + (size_t)(blockIdx.x / (kBiaRows / kRowsPerGroup)) * kPostRec +
                         blockIdx.x % (kBiaRows / kRowsPerGroup) * kRowsPerGroup;
    for (int t = threadIdx.x; t < kRowsPerGroup * per; t += kRowThreads) {
        const int r = t / per, k = 8 * (t - r * per), id = ids[r];
        if (id < 0 || k >= d) continue;
        const uint4 v = eight_of_codes(*reinterpret_cast<const uint2 *>(codes + (size_t)id * wide + k),
                                       scales[(size_t)id * (wide / kRowBlock) + k / kRowBlock]);
        uint16_t *row = x + (size_t)id * d + k;
        *reinterpret_cast<uint2 *>(row) = make_uint2(v.x, v.y);
        if (k + 4 < d) *reinterpret_cast<uint2 *>(row + 4) = make_uint2(v.z, v.w);
    }
}

}  // namespace

hipError_t launch_pack_rows(const KernelPlan &p, const uint16_t *x, int d, uint8_t *codes, uint8_t *scales,
                            hipStream_t stream) {
    hipLaunchKernelGGL(pack_rows_kernel, dim3(p.n_posts * (kBiaRows / kRowsPerGroup)), dim3(kRowThreads), 0, stream,
                       p.posts, d, x, codes, scales);
    return hipGetLastError();
}

hipError_t launch_unpack_rows(const KernelPlan &p, const uint8_t *codes, const uint8_t *scales, int d, uint16_t *x,
                              hipStream_t stream) {
    hipLaunchKernelGGL(unpack_rows_kernel, dim3(p.n_posts * (kBiaRows / kRowsPerGroup)), dim3(kRowThreads), 0, stream,
                       p.posts, d, codes, scales, x);
    return hipGetLastError();
}

}  // namespace crf
