// e4m3 values with a scale for each block of 128 (include/dsla.h): what their producers (norms.hip) share.
#pragma once
#include "dsla_internal.h"

namespace dsla {

// Blocks below this share its scale, so that neither a scale nor its inverse leaves the normal numbers.
constexpr float kLeastAmax = 0x1p-100f;
constexpr float kMostE4m3 = 448.f;

// n / d for n below 2^31 (Granlund and Montgomery's multiplication).
struct Divisor {
    uint32_t factor, shift;
    explicit Divisor(uint32_t d) : factor(0), shift(0)
    {
        while ((1ull << shift) < d) ++shift;
        factor = static_cast<uint32_t>(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return (__umulhi(n, factor) + n) >> shift; }
};

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
// The largest of them among n values: the maximum passes over NaN, and only where an infinity is among them they are looked at again.
template <int N>
__device__ __forceinline__ float largest(const float (&f)[N])
{
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) a = fmaxf(a, fabsf(f[i]));
    if (a == __builtin_inff()) {
        a = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) a = fmaxf(a, finite_magnitude(f[i]));
    }
    return a;
}

// Four values to four bytes, rounded to nearest even.  Times the inverse of their scale they are at most 448, or with fp32 scales an ulp more,
// which rounds to 448; infinities and NaN become NaN.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return static_cast<uint32_t>(w);
}

}  // namespace dsla
