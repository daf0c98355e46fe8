// crf_rows.h -- the 8-bit form of an activation row, for the kernels that
// write it and those that read it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace crf {

// Codes that share a power of two, and the codes of a row of d entries.
constexpr int kRowBlock = 32;
__host__ __device__ inline int row_codes(int d) { return (d + kRowBlock - 1) / kRowBlock * kRowBlock; }

// Two float32 as bf16, rounded to nearest even.
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// Eight e4m3 codes times 2^(scale - 127), as bf16 (exact but for results
// below bf16's smallest normal number).
__device__ __forceinline__ uint4 eight_of_codes(uint2 c, uint32_t scale) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const float s = scale ? __builtin_bit_cast(float, scale << 23) : __builtin_bit_cast(float, 0x400000u);   // 2^-127
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, true);
    const f32x2 d = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, false), e = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, true);
    return make_uint4(two_bf16(a[0] * s, a[1] * s), two_bf16(b[0] * s, b[1] * s), two_bf16(d[0] * s, d[1] * s),
                      two_bf16(e[0] * s, e[1] * s));
}

}  // namespace crf
