// Clouds held in 8-bit floating point: layout of the buffer, and the values it stands for.
//
// A cloud of [W][npts][d] points is one buffer of three parts, each on a 256-byte boundary:
//   codes   [W * npts][32 ceil(d/32)] bytes, e4m3; dimensions from d to the next multiple of 32 hold code 0
//   scales  [W * npts][4 ceil(d/512)] bytes, a power of two (e8m0) for each block of 128 dimensions; unused bytes are zero
//   norms   [W * npts] floats, the squared length of the point that codes and scales stand for
// value = e4m3 code * block scale.  Scales lie between 2^-100 and 2^120: every value has four bits of mantissa and an exponent of
// -109 or more, and is exact in fp32 and bf16.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "skb_cloud4.cuh"

namespace skb {

constexpr int CLOUD8_MAX_D = 1024, CLOUD8_BLOCK = 128, CLOUD8_MIN_E = -100, CLOUD8_MAX_E = 120;
constexpr int FMT_MX8 = 4;                    // next to SKB_MX4, SKB_NV4

struct Cloud8 {
    const uint8_t *codes, *scales;
    const float *norms;
    int cb, sb;                               // bytes of a point's codes and scales
};
__host__ __device__ inline int cloud8_code_bytes(int d) { return (d + 31) / 32 * 32; }
__host__ __device__ inline int cloud8_scale_bytes(int d) { return (d + 511) / 512 * 4; }
inline size_t cloud8_bytes(size_t rows, int d)
{
    return cloud4_pad(rows * cloud8_code_bytes(d)) + cloud4_pad(rows * cloud8_scale_bytes(d)) + cloud4_pad(rows * 4);
}
inline Cloud8 cloud8_view(const void *buf, size_t rows, int d)
{
    Cloud8 c;
    c.cb = cloud8_code_bytes(d);
    c.sb = cloud8_scale_bytes(d);
    c.codes = (const uint8_t *)buf;
    c.scales = c.codes + cloud4_pad(rows * c.cb);
    c.norms = (const float *)(c.scales + cloud4_pad(rows * c.sb));
    return c;
}

#ifdef __CUDACC__
// two codes as floats (exact)
__device__ __forceinline__ float2 e4m3_pair(uint32_t two)
{
    uint32_t h;
    asm("{\n\t.reg .b16 p;\n\tcvt.u16.u32 p, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, p;\n\t}" : "=r"(h) : "r"(two));
    float2 v;
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(v.x), "=f"(v.y) : "r"(h));
    return v;
}
#endif

}  // namespace skb
