// Sixteen consecutive dimensions of a point in and out, as the kernels that round clouds take them; exponents of floats.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace skb {

__device__ __forceinline__ uint32_t bf16_bits(float v) { return __float_as_uint(v) >> 16; }   // of values that bf16 holds exactly
__device__ __forceinline__ int exponent_of(float v)          // floor(log2 v), v > 0 finite
{
    const uint32_t b = __float_as_uint(v);
    return b >= 0x00800000u ? (int)(b >> 23) - 127 : -118 - __clz((int)b);    // (subnormal: 2^-149 * b)
}
// 2^e for -149 <= e <= 127
__device__ __forceinline__ float power_of_two(int e)
{
    return e >= -126 ? __uint_as_float((uint32_t)(e + 127) << 23) : __uint_as_float(1u << (e + 149));
}

template <bool BF16>
__device__ __forceinline__ void load16(const void *src, size_t row, int k0, int d, bool wide, float (&v)[16])
{
    const size_t at = row * d + k0;
    if (wide && k0 + 16 <= d) {
        if constexpr (BF16) {
            const uint4 *p = reinterpret_cast<const uint4 *>((const uint16_t *)src + at);
            const uint4 a = p[0], b = p[1];
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
        } else {
            const float4 *p = reinterpret_cast<const float4 *>((const float *)src + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) { const float4 a = p[i]; v[4 * i] = a.x; v[4 * i + 1] = a.y; v[4 * i + 2] = a.z; v[4 * i + 3] = a.w; }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        v[i] = 0.f;
        if (k0 + i < d) v[i] = BF16 ? __uint_as_float((uint32_t)((const uint16_t *)src)[at + i] << 16) : ((const float *)src)[at + i];
    }
}

// 16 values of a point: bf16 or fp32, in 16-byte stores where they may be
__device__ __forceinline__ void store16(void *dst, bool bf16, size_t row, int k0, int d, bool wide, const float (&v)[16])
{
    const size_t at = row * d + k0;
    if (wide && k0 + 16 <= d) {
        if (bf16) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = bf16_bits(v[2 * i]) | (bf16_bits(v[2 * i + 1]) << 16);
            uint4 *p = reinterpret_cast<uint4 *>((uint16_t *)dst + at);
            p[0] = make_uint4(w[0], w[1], w[2], w[3]);
            p[1] = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
            float4 *p = reinterpret_cast<float4 *>((float *)dst + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (k0 + i < d) {
            if (bf16) ((uint16_t *)dst)[at + i] = (uint16_t)bf16_bits(v[i]);
            else ((float *)dst)[at + i] = v[i];
        }
}

}  // namespace skb
