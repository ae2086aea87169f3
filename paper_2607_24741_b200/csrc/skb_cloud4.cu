// Clouds in microscaled 4-bit floating point: rounding to them and back (layout in skb_cloud4.cuh).
//
// Rounding, for the values v of a point:
//   mx4  blocks of 32: scale 2^(floor(log2 max|v|) - 2), so that the largest value falls into [4, 8) and what is above
//        6 is held as 6; scales are clamped to [2^-127, 2^127], a block of zeros has the smallest
//   nv4  a power of two for the point, P = 2^(floor(log2 max|v|) - 10) clamped below at 2^-126; blocks of 16 with the
//        scale max|v| / 6 / P rounded to e4m3 (at most 352 of its 448; 320 where P is 2^117, the largest there is)
//   codes are |v| / scale to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6, halves to the even code
// A point with a value that is not finite has NaN in all of its scales.
//
// Both read a cloud once and write it once, bounded by memory.  A warp takes a point of up to 512 dimensions (a part
// of a warp a shallower one), 16 consecutive dimensions to a thread: they stay in registers between the point's maximum
// and the codes, and 16 codes are one 8-byte store.  Packing with values in bf16: 64 x 1024 x 512 bf16 to mx4 28.8 us for 152 MB
// (82 % of the measured copy rate), 8 x 16384 x 512 fp32 to nv4 97 us for 440 MB (70 %: the exact quotients of nv4 fill 3.1 of
// an SM's 4 issue slots a cycle).
#include <cuda_runtime.h>
#include <string>

#include "skb_cloud4.cuh"
#include "skb_cloud_io.cuh"
#include "skb_operators.h"

namespace skb {
namespace {

constexpr int PK_WARPS = 4;

// v / b for v, b > 0, inv near 1 / b, rounded so that halves of the 4-bit grid and of e4m3 are seen for what they are: the
// quotient is cut to 24 bits and its last bit set where something was cut off ("round to odd"), after which a second
// rounding to far fewer bits is the rounding of the exact quotient.
__device__ __forceinline__ float quotient_odd(float v, float b, float inv)
{
    float q = v * inv;
    q = fmaf(fmaf(-q, b, v), inv, q);
    const float r = fmaf(-q, b, v);                 // exact: q is within an ulp
    int bits = __float_as_int(q) - (r < 0.f ? 1 : 0);
    if (r != 0.f) bits |= 1;
    return q > 0.f ? __int_as_float(bits) : 0.f;
}
// four codes as two bytes, halves to even, at most 6
__device__ __forceinline__ uint32_t e2m1x4(float a, float b, float c, float d)
{
    uint32_t out;
    asm("{\n\t.reg .b8 l, h, z;\n\tcvt.rn.satfinite.e2m1x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 h, %4, %3;\n\t"
        "cvt.u8.u32 z, 0;\n\tmov.b32 %0, {l, h, z, z};\n\t}" : "=r"(out) : "f"(a), "f"(b), "f"(c), "f"(d));
    return out;
}
__device__ __forceinline__ uint32_t e4m3_byte(float v)
{
    uint32_t out;
    asm("{\n\t.reg .b16 p;\n\tcvt.rn.satfinite.e4m3x2.f32 p, %1, %2;\n\tcvt.u32.u16 %0, p;\n\t}" : "=r"(out) : "f"(0.f), "f"(v));
    return out;
}

// LANES threads to a point, CH times 16 dimensions to each
template <bool NV, bool BF16, int LANES, int CH>
__global__ void __launch_bounds__(PK_WARPS * 32) pack_kernel(const void *src, Cloud4 out, long long rows, int d, bool wide_in,
                                                             void *values, bool values_bf16, bool wide_out)
{
    const int lane = threadIdx.x & 31, sub = lane % LANES;
    const long long row = ((long long)blockIdx.x * PK_WARPS + (threadIdx.x >> 5)) * (32 / LANES) + lane / LANES;
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
        for (int i = 0; i < 16; ++i) {
            top[c] = fmaxf(top[c], fabsf(v[c][i]));
            bad |= !(fabsf(v[c][i]) <= 3.402823466e38f);
        }
    }
    float whole = top[0];
    if constexpr (CH == 2) whole = fmaxf(whole, top[1]);
#pragma unroll
    for (int off = 1; off < LANES; off *= 2) {
        whole = fmaxf(whole, __shfl_xor_sync(0xffffffffu, whole, off));
        bad |= __shfl_xor_sync(0xffffffffu, (int)bad, off) != 0;
    }
    int pe = 0;                                                  // exponent of the point's power of two
    if (NV && whole > 0.f && !bad) pe = max(exponent_of(whole) - 10, -126);
    const float point = power_of_two(pe), point_inv = power_of_two(-pe);
    uint8_t *codes = const_cast<uint8_t *>(out.codes), *scales = const_cast<uint8_t *>(out.scales);
    const int nb16 = (d + 31) / 32 * 2;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int b16 = c * LANES + sub;
        float scale;                                             // what a code stands for, over its grid value
        uint32_t byte;
        float q[16];
        if constexpr (NV) {
            const float t = bad ? 0.f : top[c] * point_inv;
            byte = bad ? 0x7fu : e4m3_byte(quotient_odd(t, 6.f, 1.f / 6.f));
            if (pe == 117 && !bad) byte = min(byte, 0x7au);      // 320: the next scale times 6 is past fp32's range
            const float bs = e4m3_value(byte), inv = bs > 0.f ? 1.f / bs : 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float a = bs > 0.f ? quotient_odd(fabsf(v[c][i]) * point_inv, bs, inv) : 0.f;
                q[i] = copysignf(a, v[c][i]);
            }
            scale = bs * point;
        } else {
            const float other = __shfl_xor_sync(0xffffffffu, top[c], 1);
            const float t = fmaxf(top[c], other);
            const int e = t > 0.f && !bad ? max(exponent_of(t) - 2, -127) : -127;
            byte = bad ? 0xffu : (uint32_t)(e + 127);
            const float inv = power_of_two(-e);
#pragma unroll
            for (int i = 0; i < 16; ++i) q[i] = v[c][i] * inv;   // exact
            scale = bad ? __uint_as_float(0x7fffffffu) : power_of_two(e);
        }
        uint32_t w[2] = {0u, 0u};
        if (!bad)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i / 2] |= e2m1x4(q[4 * i], q[4 * i + 1], q[4 * i + 2], q[4 * i + 3]) << (16 * (i & 1));
        if (!live || b16 >= nb16) continue;
        *reinterpret_cast<uint2 *>(codes + (size_t)row * out.cb + 8 * b16) = make_uint2(w[0], w[1]);
        if (NV) scales[(size_t)row * out.sb + b16] = (uint8_t)byte;
        else if (!(b16 & 1)) scales[(size_t)row * out.sb + (b16 >> 1)] = (uint8_t)byte;
        if (values) {
            float r[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 p = e2m1_pair((w[i / 4] >> (8 * (i & 3))) & 255u);
                r[2 * i] = p.x * scale;
                r[2 * i + 1] = p.y * scale;
            }
            if (16 * b16 < d) store16(values, values_bf16, (size_t)row, 16 * b16, d, wide_out, r);
        }
    }
    if (live && sub == 0) {
        for (int i = NV ? nb16 : nb16 / 2; i < out.sb; ++i) scales[(size_t)row * out.sb + i] = 0;
        if (NV) const_cast<float *>(out.points)[row] = point;
    }
}

// 16 consecutive dimensions to a thread
__global__ void __launch_bounds__(256) unpack_kernel(Cloud4 in, long long rows, int d, void *values, bool bf16, bool wide)
{
    const int nb16 = (d + 15) / 16;
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= rows * nb16) return;
    const long long row = at / nb16;
    const int k0 = (int)(at % nb16) * 16;
    const uint2 w = *reinterpret_cast<const uint2 *>(in.codes + (size_t)row * in.cb + k0 / 2);
    const float scale = cloud4_scale(in, (size_t)row, k0);
    float r[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 p = e2m1_pair(((i < 4 ? w.x : w.y) >> (8 * (i & 3))) & 255u);
        r[2 * i] = p.x * scale;
        r[2 * i + 1] = p.y * scale;
    }
    store16(values, bf16, (size_t)row, k0, d, wide, r);
}

template <bool NV, bool BF16, int LANES, int CH>
void launch_pack(const void *v, const Cloud4 &out, long long rows, int d, void *values, bool values_bf16, cudaStream_t st)
{
    const int per_block = PK_WARPS * (32 / LANES);
    const bool wide_in = (uintptr_t)v % 16 == 0 && d * (BF16 ? 2 : 4) % 16 == 0;
    const bool wide_out = (uintptr_t)values % 16 == 0 && d * (values_bf16 ? 2 : 4) % 16 == 0;
    pack_kernel<NV, BF16, LANES, CH><<<(unsigned)((rows + per_block - 1) / per_block), PK_WARPS * 32, 0, st>>>(
        v, out, rows, d, wide_in, values, values_bf16, wide_out);
}
template <bool NV, bool BF16>
void pack_by_depth(const void *v, const Cloud4 &out, long long rows, int d, void *values, bool vb, cudaStream_t st)
{
    if (d <= 32) launch_pack<NV, BF16, 2, 1>(v, out, rows, d, values, vb, st);
    else if (d <= 64) launch_pack<NV, BF16, 4, 1>(v, out, rows, d, values, vb, st);
    else if (d <= 128) launch_pack<NV, BF16, 8, 1>(v, out, rows, d, values, vb, st);
    else if (d <= 256) launch_pack<NV, BF16, 16, 1>(v, out, rows, d, values, vb, st);
    else if (d <= 512) launch_pack<NV, BF16, 32, 1>(v, out, rows, d, values, vb, st);
    else launch_pack<NV, BF16, 32, 2>(v, out, rows, d, values, vb, st);
}

}  // namespace

const char *cloud4_refused(int W, int npts, int d, int format)
{
    if (format != FMT_MX4 && format != FMT_NV4) return "format must be SKB_MX4 or SKB_NV4";
    if (W < 1 || npts < 1 || d < 1) return "W, the number of points and d must be >= 1";
    if (d > CLOUD4_MAX_D) return "d must be at most 1024";
    if ((long long)W * npts > 0x7fffffffLL) return "more than 2^31 - 1 points";
    return nullptr;
}

thread_local std::string op_error;
skb_status op_fail(skb_status st, const std::string &msg) { op_error = msg; return st; }
skb_status op_launched(const char *what)
{
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return op_fail(SKB_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
    op_error.clear();
    return SKB_OK;
}

}  // namespace skb

using namespace skb;

extern "C" const char *sinkhorn_operator_last_error(void) { return op_error.c_str(); }

extern "C" size_t sinkhorn_cloud4_bytes(int W, int npts, int d, int format)
{
    return cloud4_refused(W, npts, d, format) ? 0 : cloud4_bytes((size_t)W * npts, d, format);
}

extern "C" skb_status sinkhorn_cloud4_pack(const void *v, int v_dtype, int W, int npts, int d, int format, void *cloud,
                                           void *values, int values_dtype, void *stream)
{
    if (!v || !cloud) return op_fail(SKB_ERR_NULL, "v and cloud are required");
    if (const char *why = cloud4_refused(W, npts, d, format)) return op_fail(SKB_ERR_SHAPE, why);
    if (v_dtype != SKB_F32 && v_dtype != SKB_BF16) return op_fail(SKB_ERR_VALUE, "v must be SKB_F32 or SKB_BF16");
    if (values && values_dtype != SKB_F32 && values_dtype != SKB_BF16) return op_fail(SKB_ERR_VALUE, "values must be SKB_F32 or SKB_BF16");
    if ((uintptr_t)cloud % 256) return op_fail(SKB_ERR_WORKSPACE, "cloud must be 256-byte aligned");
    const long long rows = (long long)W * npts;
    const Cloud4 out = cloud4_view(cloud, (size_t)rows, d, format);
    const bool vb = values_dtype == SKB_BF16;
    cudaStream_t st = (cudaStream_t)stream;
    if (format == SKB_NV4) {
        if (v_dtype == SKB_BF16) pack_by_depth<true, true>(v, out, rows, d, values, vb, st);
        else pack_by_depth<true, false>(v, out, rows, d, values, vb, st);
    } else {
        if (v_dtype == SKB_BF16) pack_by_depth<false, true>(v, out, rows, d, values, vb, st);
        else pack_by_depth<false, false>(v, out, rows, d, values, vb, st);
    }
    return op_launched("cloud4_pack");
}

extern "C" skb_status sinkhorn_cloud4_unpack(const void *cloud, int W, int npts, int d, int format, void *values, int values_dtype, void *stream)
{
    if (!cloud || !values) return op_fail(SKB_ERR_NULL, "cloud and values are required");
    if (const char *why = cloud4_refused(W, npts, d, format)) return op_fail(SKB_ERR_SHAPE, why);
    if (values_dtype != SKB_F32 && values_dtype != SKB_BF16) return op_fail(SKB_ERR_VALUE, "values must be SKB_F32 or SKB_BF16");
    if ((uintptr_t)cloud % 256) return op_fail(SKB_ERR_WORKSPACE, "cloud must be 256-byte aligned");
    const long long rows = (long long)W * npts, threads = rows * ((d + 15) / 16);
    const bool bf16 = values_dtype == SKB_BF16, wide = (uintptr_t)values % 16 == 0 && d * (bf16 ? 2 : 4) % 16 == 0;
    unpack_kernel<<<(unsigned)((threads + 255) / 256), 256, 0, (cudaStream_t)stream>>>(cloud4_view(cloud, (size_t)rows, d, format), rows, d, values, bf16, wide);
    return op_launched("cloud4_unpack");
}
