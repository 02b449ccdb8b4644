// e4m3 values with a scale for each block of 128 (include/dsla.h): what their producers (norms.hip) share.
#pragma once
#include "dsla_internal.h"

namespace dsla {

// Blocks below this share its scale, so that neither a scale nor its inverse leaves the normal numbers.
constexpr float kLeastAmax = 0x1p-100f;
constexpr float kMostE4m3 = 448.f;

__host__ __device__ __forceinline__ int scale_pitch(int cols) { return DSLA_SCALE_PITCH(cols); }

// A block's scale from its largest finite magnitude: what is stored, and what values are multiplied by.  E8M0: 448 = 1.75 * 2^8, so
// the least power of two that keeps amax = m 2^E (1 <= m < 2) within it is 2^(E - 8), or twice that where m > 1.75.
template <bool E8M0>
struct BlockScale {
    uint32_t stored;   // fp32 bits, or the byte
    float inverse;
    __device__ __forceinline__ explicit BlockScale(float amax)
    {
        amax = fmaxf(amax, kLeastAmax);
        if (E8M0) {
            const uint32_t bits = __float_as_uint(amax);
            stored = (bits >> 23) - 8u + ((bits & 0x7fffffu) > 0x600000u ? 1u : 0u);
            inverse = __uint_as_float((254u - stored) << 23);
        } else {
            stored = __float_as_uint(amax / kMostE4m3);
            inverse = kMostE4m3 / amax;
        }
    }
    __device__ __forceinline__ void store(void *scales, size_t at) const
    {
        if (E8M0) static_cast<uint8_t *>(scales)[at] = static_cast<uint8_t>(stored);
        else static_cast<uint32_t *>(scales)[at] = stored;
    }
};

// The magnitude that counts for a block's scale.
__device__ __forceinline__ float finite_magnitude(float x)
{
    const float a = fabsf(x);
    return a < __builtin_inff() ? a : 0.f;   // (NaN: 0)
}

// x / scale as e4m3 sees it: at most 448 (the product may be an ulp above), NaN for what was not finite.
__device__ __forceinline__ float in_range(float x, float inverse)
{
    const float v = x * inverse;
    return fabsf(v) < 512.f ? fminf(fmaxf(v, -kMostE4m3), kMostE4m3) : __builtin_nanf("");
}

// Four values to four bytes, rounded to nearest even.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return static_cast<uint32_t>(w);
}

}  // namespace dsla
