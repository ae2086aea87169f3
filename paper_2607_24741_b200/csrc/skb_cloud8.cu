// Clouds in 8-bit floating point: rounding to them and back (layout in skb_cloud8.cuh).
//
// Rounding, for the values v of a block of 128 dimensions of a point:
//   scale  2^E, E the smallest integer from -100 on with max|v| <= 448 * 2^E (448 is the largest code): nothing saturates
//   codes  v / scale to the nearest of e4m3, halves to the even code (240 at most where E is 120: no value passes fp32's range)
// A power of two and not max|v| / 448: e4m3 has its three bits of mantissa wherever in its range a value lies, so the other scale would
// not round any better, but for values below 2^-14 of the largest; and this one leaves values exact in bf16 and is what the
// block-scaled matrix instructions take.  A point with a value that is not finite becomes NaN as a whole.
//
// Both read a cloud once and write it once.  64 x 1024 x 512 from bf16, with the values in bf16 (168 MB), take 30.8 us, 83 % of the measured copy rate
// (34.8 with a comparison of every value for what is not finite, and one for what would saturate).  Sixteen consecutive dimensions to a thread, eight threads to a block, up to
// a warp to a point: values stay in registers between the block's maximum and the codes, and 16 codes are one 16-byte store.
// The way back takes 19.0 us to bf16 (101 MB, 81 % of the copy rate) and 39.9 to fp32 (168 MB, 64 %).
#include <cuda_runtime.h>
#include <string>

#include "skb_cloud8.cuh"
#include "skb_cloud_io.cuh"
#include "skb_operators.h"

namespace skb {
namespace {

constexpr int P8_WARPS = 4;

__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d)
{
    uint32_t out;
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(out) : "f"(a), "f"(b), "f"(c), "f"(d));
    return out;
}

// the larger of two, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// LANES threads to a point, CH times 16 dimensions to each
template <bool BF16, int LANES, int CH>
__global__ void __launch_bounds__(P8_WARPS * 32) pack8_kernel(const void *src, Cloud8 out, long long rows, int d, bool wide_in,
                                                              void *values, bool values_bf16, bool wide_out)
{
    constexpr int BLOCK_LANES = LANES < 8 ? LANES : 8;
    const int lane = threadIdx.x & 31, sub = lane % LANES;
    const long long row = ((long long)blockIdx.x * P8_WARPS + (threadIdx.x >> 5)) * (32 / LANES) + lane / LANES;
    const bool live = row < rows;
    float v[CH][16], top[CH];
    bool bad = false;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int k0 = (c * LANES + sub) * 16;
#pragma unroll
        for (int i = 0; i < 16; ++i) v[c][i] = 0.f;
        if (live && k0 < d) load16<BF16>(src, (size_t)row, k0, d, wide_in, v[c]);
        top[c] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) top[c] = max_nan(top[c], fabsf(v[c][i]));
#pragma unroll
        for (int off = 1; off < BLOCK_LANES; off *= 2) top[c] = max_nan(top[c], __shfl_xor_sync(0xffffffffu, top[c], off));
        bad |= !(top[c] <= 3.402823466e38f);
    }
#pragma unroll
    for (int off = BLOCK_LANES; off < LANES; off *= 2) bad |= __shfl_xor_sync(0xffffffffu, (int)bad, off) != 0;
    uint8_t *codes = const_cast<uint8_t *>(out.codes), *scales = const_cast<uint8_t *>(out.scales);
    double norm = 0.0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at16 = c * LANES + sub, k0 = 16 * at16;
        int e = CLOUD8_MIN_E;
        if (top[c] > 0.f && !bad) {
            e = max(exponent_of(top[c]) - 8, CLOUD8_MIN_E);
            if (top[c] > 448.f * power_of_two(e)) ++e;
        }
        const float inv = power_of_two(-e);
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        if (e == CLOUD8_MAX_E)
#pragma unroll
            for (int i = 0; i < 16; ++i) v[c][i] = fminf(fmaxf(v[c][i], -240.f * 0x1p120f), 240.f * 0x1p120f);
        if (!bad)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = e4m3x4(v[c][4 * i] * inv, v[c][4 * i + 1] * inv, v[c][4 * i + 2] * inv, v[c][4 * i + 3] * inv);
        float r[16], s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 p = e4m3_pair((w[i / 2] >> (16 * (i & 1))) & 0xffffu);
            s = fmaf(p.x, p.x, fmaf(p.y, p.y, s));                // squares of four bits: each exact
            r[2 * i] = p.x;
            r[2 * i + 1] = p.y;
        }
        const double scale = bad ? __longlong_as_double(0x7ff8000000000000LL) : (double)power_of_two(e);
        norm += (double)s * scale * scale;
        if (!live || k0 >= d + 31 - (d + 31) % 32) continue;
        *reinterpret_cast<uint4 *>(codes + (size_t)row * out.cb + k0) = make_uint4(w[0], w[1], w[2], w[3]);
        if (at16 % 8 == 0) scales[(size_t)row * out.sb + at16 / 8] = bad ? 255 : (uint8_t)(e + 127);
        if (values && k0 < d) {
            const float f = bad ? __uint_as_float(0x7fffffffu) : power_of_two(e);
#pragma unroll
            for (int i = 0; i < 16; ++i) r[i] *= f;
            store16(values, values_bf16, (size_t)row, k0, d, wide_out, r);
        }
    }
#pragma unroll
    for (int off = 1; off < LANES; off *= 2) norm += __shfl_xor_sync(0xffffffffu, norm, off);
    if (live && sub == 0) {
        for (int i = (d + CLOUD8_BLOCK - 1) / CLOUD8_BLOCK; i < out.sb; ++i) scales[(size_t)row * out.sb + i] = 0;
        const_cast<float *>(out.norms)[row] = (float)norm;
    }
}

// 16 consecutive dimensions to a thread
__global__ void __launch_bounds__(256) unpack8_kernel(Cloud8 in, long long rows, int d, void *values, bool bf16, bool wide)
{
    const int nb16 = (d + 15) / 16;
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= rows * nb16) return;
    const long long row = at / nb16;
    const int k0 = (int)(at % nb16) * 16;
    const uint4 w = *reinterpret_cast<const uint4 *>(in.codes + (size_t)row * in.cb + k0);
    const float scale = e8m0_value(in.scales[(size_t)row * in.sb + k0 / CLOUD8_BLOCK]);
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
    float r[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 p = e4m3_pair((word[i / 2] >> (16 * (i & 1))) & 0xffffu);
        r[2 * i] = p.x * scale;
        r[2 * i + 1] = p.y * scale;
    }
    store16(values, bf16, (size_t)row, k0, d, wide, r);
}

template <bool BF16, int LANES, int CH>
void launch_pack8(const void *v, const Cloud8 &out, long long rows, int d, void *values, bool values_bf16, cudaStream_t st)
{
    const int per_block = P8_WARPS * (32 / LANES);
    const bool wide_in = (uintptr_t)v % 16 == 0 && d * (BF16 ? 2 : 4) % 16 == 0;
    const bool wide_out = (uintptr_t)values % 16 == 0 && d * (values_bf16 ? 2 : 4) % 16 == 0;
    pack8_kernel<BF16, LANES, CH><<<(unsigned)((rows + per_block - 1) / per_block), P8_WARPS * 32, 0, st>>>(
        v, out, rows, d, wide_in, values, values_bf16, wide_out);
}
template <bool BF16>
void pack8_by_depth(const void *v, const Cloud8 &out, long long rows, int d, void *values, bool vb, cudaStream_t st)
{
    if (d <= 32) launch_pack8<BF16, 2, 1>(v, out, rows, d, values, vb, st);
    else if (d <= 64) launch_pack8<BF16, 4, 1>(v, out, rows, d, values, vb, st);
    else if (d <= 128) launch_pack8<BF16, 8, 1>(v, out, rows, d, values, vb, st);
    else if (d <= 256) launch_pack8<BF16, 16, 1>(v, out, rows, d, values, vb, st);
    else if (d <= 512) launch_pack8<BF16, 32, 1>(v, out, rows, d, values, vb, st);
    else launch_pack8<BF16, 32, 2>(v, out, rows, d, values, vb, st);
}

}  // namespace

const char *cloud8_refused(int W, int npts, int d)
{
    if (W < 1 || npts < 1 || d < 1) return "W, the number of points and d must be >= 1";
    if (d > CLOUD8_MAX_D) return "d must be at most 1024";
    if ((long long)W * npts > 0x7fffffffLL) return "more than 2^31 - 1 points";
    return nullptr;
}

}  // namespace skb

using namespace skb;

extern "C" size_t sinkhorn_cloud8_bytes(int W, int npts, int d)
{
    return cloud8_refused(W, npts, d) ? 0 : cloud8_bytes((size_t)W * npts, d);
}

extern "C" skb_status sinkhorn_cloud8_pack(const void *v, int v_dtype, int W, int npts, int d, void *cloud, void *values, int values_dtype,
                                           void *stream)
{
    if (!v || !cloud) return op_fail(SKB_ERR_NULL, "v and cloud are required");
    if (const char *why = cloud8_refused(W, npts, d)) return op_fail(SKB_ERR_SHAPE, why);
    if (v_dtype != SKB_F32 && v_dtype != SKB_BF16) return op_fail(SKB_ERR_VALUE, "v must be SKB_F32 or SKB_BF16");
    if (values && values_dtype != SKB_F32 && values_dtype != SKB_BF16) return op_fail(SKB_ERR_VALUE, "values must be SKB_F32 or SKB_BF16");
    if ((uintptr_t)cloud % 256) return op_fail(SKB_ERR_WORKSPACE, "cloud must be 256-byte aligned");
    if ((uintptr_t)v % (v_dtype == SKB_BF16 ? 2 : 4) || (uintptr_t)values % (values_dtype == SKB_BF16 ? 2 : 4))
        return op_fail(SKB_ERR_WORKSPACE, "v and values must be aligned to their type");
    const long long rows = (long long)W * npts;
    const Cloud8 out = cloud8_view(cloud, (size_t)rows, d);
    const bool vb = values_dtype == SKB_BF16;
    if (v_dtype == SKB_BF16) pack8_by_depth<true>(v, out, rows, d, values, vb, (cudaStream_t)stream);
    else pack8_by_depth<false>(v, out, rows, d, values, vb, (cudaStream_t)stream);
    return op_launched("cloud8_pack");
}

extern "C" skb_status sinkhorn_cloud8_unpack(const void *cloud, int W, int npts, int d, void *values, int values_dtype, void *stream)
{
    if (!cloud || !values) return op_fail(SKB_ERR_NULL, "cloud and values are required");
    if (const char *why = cloud8_refused(W, npts, d)) return op_fail(SKB_ERR_SHAPE, why);
    if (values_dtype != SKB_F32 && values_dtype != SKB_BF16) return op_fail(SKB_ERR_VALUE, "values must be SKB_F32 or SKB_BF16");
    if ((uintptr_t)cloud % 256) return op_fail(SKB_ERR_WORKSPACE, "cloud must be 256-byte aligned");
    const bool bf16 = values_dtype == SKB_BF16, wide = (uintptr_t)values % 16 == 0 && d * (bf16 ? 2 : 4) % 16 == 0;
    if ((uintptr_t)values % (bf16 ? 2 : 4)) return op_fail(SKB_ERR_WORKSPACE, "values must be aligned to their type");
    // (2^31 - 1 points of 1024 dimensions are 2^29 blocks of 256 threads)
    const long long rows = (long long)W * npts, threads = rows * ((d + 15) / 16);
    unpack8_kernel<<<(unsigned)((threads + 255) / 256), 256, 0, (cudaStream_t)stream>>>(cloud8_view(cloud, (size_t)rows, d), rows, d, values, bf16, wide);
    return op_launched("cloud8_unpack");
}

extern "C" skb_status sinkhorn_cloud8_dots(const void *x, const void *y, int W, int n, int m, int d, float *out, void *stream)
{
    if (!x || !y || !out) return op_fail(SKB_ERR_NULL, "x, y and out are required");
    if (const char *why = cloud8_refused(W, n, d)) return op_fail(SKB_ERR_SHAPE, why);
    if (const char *why = cloud8_refused(W, m, d)) return op_fail(SKB_ERR_SHAPE, why);
    if ((uintptr_t)x % 256 || (uintptr_t)y % 256) return op_fail(SKB_ERR_WORKSPACE, "x and y must be 256-byte aligned");
    if ((uintptr_t)out % 4) return op_fail(SKB_ERR_WORKSPACE, "out must be 4-byte aligned");
    const Cloud8 a = cloud8_view(x, (size_t)W * n, d), b = cloud8_view(y, (size_t)W * m, d);
    return launch_dots({a.codes, a.scales, nullptr, a.cb, a.sb}, {b.codes, b.scales, nullptr, b.cb, b.sb}, FMT_MX8, W, n, m, out, m, (cudaStream_t)stream);
}
