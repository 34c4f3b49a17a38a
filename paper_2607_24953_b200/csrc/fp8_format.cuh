// The two 8-bit formats in FP32 arithmetic: E4M3 codes with an FP32 scale for 128 elements, and with a UE8M0 scale for 32 (MXFP8).
#pragma once

#include "quant_device.cuh"

namespace fp4q {

constexpr float kFp8Top = 448.0f;              // the largest E4M3 number
constexpr float kFp8Least = 0x1p-100f;         // the least maximum that a block is scaled by, so that neither factor leaves FP32's normal range

// What the elements of a block with the largest finite magnitude m are multiplied by, and the scale that goes with it.
__device__ __forceinline__ float fp8_factor(float m) { return __fdiv_rn(kFp8Top, fmaxf(m, kFp8Least)); }
__device__ __forceinline__ float fp8_scale(float m) { return __fdiv_rn(fmaxf(m, kFp8Least), kFp8Top); }

__device__ __forceinline__ bool is_infinite(float v) { return (__float_as_uint(v) & 0x7FFFFFFFu) == 0x7F800000u; }
__device__ __forceinline__ float nan32() { return __uint_as_float(0x7FFFFFFFu); }
// |v|, or 0 where v is not finite.
__device__ __forceinline__ float finite_size(float v) { const float a = fabsf(v); return a < __uint_as_float(0x7F800000u) ? a : 0.f; }

// Code of the smallest power of two S with 448 S >= m, m finite: S = 2^(code - 127), not below 2^-127.
__device__ __forceinline__ int mx_scale_code(float m)
{
    const uint32_t b = __float_as_uint(m);
    const int c = (int)(b >> 23) - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return b < 0x00800000u || c < 0 ? 0 : c;
}

// 16 elements times `factor` as codes.  `careful`: infinities among them, which become NaN (the conversion takes them for the largest number).
__device__ __forceinline__ uint4 fp8_codes(const float (&v)[16], float factor, bool careful)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; j++) x[j] = careful && is_infinite(v[4 * i + j]) ? nan32() : v[4 * i + j] * factor;
        w[i] = cvt_rn_e4m3x4(x[3], x[2], x[1], x[0]);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace fp4q
