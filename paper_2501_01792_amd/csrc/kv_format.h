// The element formats of the paged K/V cache (FMT as in the C ABI: 0 the 16-bit storage type, 1 int8, 2 e4m3 in its OCP form)
// and the conversions between their codes and the 16-bit types.
//
// A row of dh elements has one scale: x = scale * code, scale = max(max |x| / Q, 2^-100).  Q is the largest code (127, 448), so
// that nothing saturates and an element is off by half a step at most: scale / 2 for int8, a sixteenth of the element (or
// half of 2^-9 scale) for e4m3.  The floor keeps the scale's reciprocal and its exponent representable; it makes a row of zeros
// zeros and changes a value only below 127 * 2^-100.  Every int8 and e4m3 code is exact in fp16 (and in bf16).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elem.h"

namespace hk {
namespace kvfmt {

constexpr int k16 = 0, kInt8 = 1, kE4m3 = 2;
constexpr float kLeastScale = 0x1p-100f;

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

template <int FMT>
__device__ __forceinline__ constexpr float most() { return FMT == kInt8 ? 127.f : 448.f; }

// 8 elements of a row -> 8 codes.  scale is finite and not below kLeastScale, inv = 1 / scale (rounded correctly, as the
// language's division is).  x / scale rounded correctly comes from two multiply-adds on x inv, its residue times inv added on: the
// last steps of a division, without the scaling that keeps a general one out of the ranges that cannot occur here.  (A
// residue below fp32's normal numbers is off by 2^-150 at most: 2^-50 of a code at the least scale.)
template <int FMT>
__device__ __forceinline__ u32x2_t encode8(const float (&x)[8], float scale, float inv)
{
    u32x2_t code;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float q = x[4 * w + j] * inv;
            y[j] = __builtin_fmaf(__builtin_fmaf(-q, scale, x[4 * w + j]), inv, q);
        }
        if constexpr (FMT == kInt8) {
            // |y| <= 127 up to the quotient's rounding; at 1.5 * 2^23 a float's last bit is one, so the sum rounds to nearest
            // even and its low byte is the code
            uint32_t b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = __builtin_bit_cast(uint32_t, y[j] + 12582912.f);
            code[w] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
        } else {
            const int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
            code[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], v, true);
        }
    }
    return code;
}

// 4 codes -> 4 floats.
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t code, float (&x)[4])
{
    if constexpr (FMT == kInt8) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = (float)(int8_t)(code >> (8 * j));
    } else {
        typedef float f2 __attribute__((ext_vector_type(2)));
        const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)code, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)code, true);
        x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
    }
}

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));

// Codes of bytes 2 HI, 2 HI + 1 of a word as fp16.  int8: the word has had every sign bit flipped (code + 128 as an unsigned
// byte), 0x6400 + u is the fp16 number 1024 + u.
template <int FMT, bool HI>
__device__ __forceinline__ half2_t pair_f16(uint32_t code)
{
    if constexpr (FMT == kInt8) {
        const uint32_t u = __builtin_amdgcn_perm(0x64646464u, code, HI ? 0x04030402u : 0x04010400u);
        return __builtin_bit_cast(half2_t, u) - half2_t{(_Float16)1152.f, (_Float16)1152.f};
    } else {
        return __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)code, 1.f, HI));
    }
}
template <int FMT>
__device__ __forceinline__ uint32_t biased(uint32_t code) { return FMT == kInt8 ? code ^ 0x80808080u : code; }

}  // namespace kvfmt
}  // namespace hk
