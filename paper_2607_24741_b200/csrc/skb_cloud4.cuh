// Clouds held in microscaled 4-bit floating point: layout of the buffer, and the values it stands for.
//
// A cloud of [W][npts][d] points is one buffer of three parts, each on a 256-byte boundary:
//   codes   [W * npts][16 ceil(d/32)] bytes, two e2m1 codes to a byte, the even dimension in the low half;
//           dimensions from d to the next multiple of 32 hold code 0
//   scales  [W * npts][sb] bytes, one for each block of 32 (mx4: a power of two, e8m0) or 16 dimensions (nv4: e4m3),
//           sb being their number rounded up to whole 32-bit words; unused bytes are zero
//   points  nv4 only: [W * npts] floats, a power of two for each point
// value = e2m1 code * block scale (* point's power of two).  It has at most six bits of mantissa: exact in fp32, and in
// bf16 from 2^-126 on.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace skb {

constexpr int CLOUD4_MAX_D = 1024;
constexpr int FMT_MX4 = 2, FMT_NV4 = 3;      // as SKB_MX4, SKB_NV4

struct Cloud4 {
    const uint8_t *codes, *scales;
    const float *points;                      // null for mx4
    int cb, sb;                               // bytes of a point's codes and scales
};
__host__ __device__ inline int cloud4_code_bytes(int d) { return (d + 31) / 32 * 16; }
__host__ __device__ inline int cloud4_blocks(int d, int fmt) { return (d + 31) / 32 * (fmt == FMT_NV4 ? 2 : 1); }
__host__ __device__ inline int cloud4_scale_bytes(int d, int fmt) { return (cloud4_blocks(d, fmt) + 3) / 4 * 4; }
inline size_t cloud4_pad(size_t b) { return (b + 255) / 256 * 256; }
inline size_t cloud4_bytes(size_t rows, int d, int fmt)
{
    return cloud4_pad(rows * cloud4_code_bytes(d)) + cloud4_pad(rows * cloud4_scale_bytes(d, fmt)) + (fmt == FMT_NV4 ? cloud4_pad(rows * 4) : 0);
}
inline Cloud4 cloud4_view(const void *buf, size_t rows, int d, int fmt)
{
    Cloud4 c;
    c.cb = cloud4_code_bytes(d);
    c.sb = cloud4_scale_bytes(d, fmt);
    c.codes = (const uint8_t *)buf;
    c.scales = c.codes + cloud4_pad(rows * c.cb);
    c.points = fmt == FMT_NV4 ? (const float *)(c.scales + cloud4_pad(rows * c.sb)) : nullptr;
    return c;
}

#ifdef __CUDACC__
// e2m1 codes as floats (exact): a code's exponent and mantissa are those of a float whose exponent counts from 126 less.
__device__ __forceinline__ float e2m1_value(uint32_t code)
{
    return __uint_as_float((code & 7u) << 22 | (code & 8u) << 28) * 8.507059173023462e37f;
}
// the two of a byte
__device__ __forceinline__ float2 e2m1_pair(uint32_t byte) { return make_float2(e2m1_value(byte), e2m1_value(byte >> 4)); }
__device__ __forceinline__ float e8m0_value(uint32_t b)
{
    return b == 255u ? __uint_as_float(0x7fffffffu) : b == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(b << 23);
}
__device__ __forceinline__ float e4m3_value(uint32_t b)
{
    uint32_t h;
    asm("{\n\t.reg .b16 p;\n\tcvt.u16.u32 p, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, p;\n\t}" : "=r"(h) : "r"(b & 255u));
    float v;
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.f32.f16 %0, a;\n\t}" : "=f"(v) : "r"(h));
    return v;
}
// what the block of dimension k of a point is multiplied by
__device__ __forceinline__ float cloud4_scale(const Cloud4 &c, size_t row, int k)
{
    if (c.points) return e4m3_value(c.scales[row * c.sb + (k >> 4)]) * c.points[row];
    return e8m0_value(c.scales[row * c.sb + (k >> 5)]);
}
__device__ __forceinline__ float cloud4_value(const Cloud4 &c, size_t row, int k)
{
    return e2m1_value((uint32_t)c.codes[row * c.cb + (k >> 1)] >> (4 * (k & 1))) * cloud4_scale(c, row, k);
}
#endif

}  // namespace skb
