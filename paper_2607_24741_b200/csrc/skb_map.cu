// Images of query points under the entropic map of a target cloud held in 8 bits: attention over a stored bank,
//      out_i = sum_j w_ij v_j,   w_i = softmax over j of (g_j - |x_i - y_j|^2) / eps,
// in one pass over the bank: exponents as k (2 x.y + g_j - |y_j|^2), k = log2(e) / eps, against a running maximum (|x_i|^2 is the same for all j).
//
// map_rows_kernel, here: few queries, the serving form.  Eight or sixteen queries and a part of a lane's bank to a block.  Bounded by memory: every code is
// read once (by one block of queries), and the tensor cores take the codes as they are:
//   scores   S^T = Y . X^T, 128 targets of a tile by the queries: kind::mxf8f6f4 on the codes with the blocks' powers of two as scales.  A query is a sum
//            of three e4m3 numbers a value, each a sixteenth of the one before it, with a power of two for each 128 dimensions: rounded to four bits, what is
//            left of bf16's eight, and what is left of that for values below 2^-14 of the block's largest; what remains is below 2^-26 of that.  The three are
//            rows of their own, added in fp32.  The matrix unit cuts each of an instruction's 32 products and the sum so far at 2^-25 of the largest, the result at
//            24 bits: 33 2^-25 + 2^-23 < 2^-19.8 of the magnitudes for every 32 dimensions, which is what exponents are good to
//   softmax  a thread to a target: exponentials in fp32 against the tile's maximum of the query, which carries over to a running one in fp32
//   images   O^T = V^T . P^T, 128 dimensions by the queries: kind::f8f6f4 on the codes, in the same place of shared memory, now the operand whose rows lie
//            next to each other (M-major).  Weights times the values' powers of two are two e4m3 numbers (eight bits; what is below 2^-22 of the reference is
//            lost), rows of their own again.  The reference is the tile's largest power of two, or where these are far apart the query's largest product
// so that nothing of a code passes through a register.  The same work by mma.sync, codes made f16 in registers, was bound by its instructions: one query
// to each of 8 banks of 16384 x 512 took 41 us.
// That call takes 28 us for 69 MB now, twelve queries to each of 32 banks of 8192 x 128 with values of 64 dimensions 31 us for 54 MB.  Of the first some
// 17 us are a block's time, whose tiles go by at the rate of the memory (2600 cycles for 64 KB) between the first one's arrival (some 8000, as all of a
// block's slots are asked for at once) and the last one's way through the roles (scores 500, softmax 2000, images 1000, results 2000); with twelve queries
// the softmax takes 1.5 times as long as the memory.  Made no difference: loads that start before the block is ready, a softmax
// against a whole number that is seldom raised instead of the tile's maximum, a third group of warps for it, terms brought into L2 ahead.
//   warps 0-3   softmax, and 12-15 where registers allow: every other tile each
//   warps 4-7   images: tensor memory -> fp32 sums in registers, a thread to a dimension of every 128
//   warp 8      loads by TMA: slots of 128 targets by 128 dimensions (16 KB, 128-byte swizzle, targets past the end are zeros)
//   warp 9      scores' matrix instructions, warp 11 the images': either waits for what it needs
//   warp 10     targets' scales and terms, up to six tiles ahead; a second such warp, where registers allow, every other tile each
// Several blocks that share a lane's bank leave (maximum, sum, image), which map_join_kernel adds up.  Every wait is bounded (skb_tmem.cuh): one that
// runs out ends all roles, and the block's images are NaN.
#include <cuda.h>
#include <cuda_runtime.h>
#include <string>

#include "skb_cloud_io.cuh"
#include "skb_f32x2.cuh"
#include "skb_map.cuh"
#include "skb_operators.h"
#include "skb_tmem.cuh"

namespace skb {
namespace {

constexpr int MR_T = 128;                                     // points of a tile
constexpr uint32_t MR_SLOT = MR_T * 128;
constexpr int MR_MAX_SLOTS = 16, MR_MAX_BLOCKS = 8, MR_AHEAD = 6;     // MR_AHEAD: tiles whose scales and terms are there at once
constexpr int MR_SPREAD = 3;                                  // how far apart values' powers of two of a tile may be for their largest to be all weights' reference
// rows of the queries' operand: three numbers of each query, and how many rows the instruction takes
template <int NQ> constexpr int MR_ROWS = NQ == 8 ? 32 : 48;
template <int NQ> constexpr int MR_SCOLS = NQ == 8 ? 32 : 64;  // columns of tensor memory that its result takes

__device__ __forceinline__ uint32_t e4m3_two(float lo, float hi)
{
    uint32_t r;
    asm("{\n\t.reg .b16 p;\n\tcvt.rn.satfinite.e4m3x2.f32 p, %2, %1;\n\tcvt.u32.u16 %0, p;\n\t}" : "=r"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void tma_points(uint32_t dst, const CUtensorMap *tm, int byte, int point, int lane, uint32_t mbar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(byte), "r"(point), "r"(lane), "r"(mbar) : "memory");
}
// 128 rows' words of four scales, 512 bytes of shared memory, into four columns of tensor memory
__device__ __forceinline__ void scales_in(uint32_t taddr, uint32_t saddr)
{
    const uint64_t desc = (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(128u >> 4) << 32) | (1ull << 46);
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb) : "memory");
}
__device__ __forceinline__ void mma_codes(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// warps of the softmax: two groups of four that take turns, where registers allow
template <int NQ, int UNITS> constexpr int MR_GROUPS = NQ * UNITS <= 32 ? 2 : 1;
// warps for the targets' terms: one takes as long for a tile as all else of it (two: one query to 8 banks of 16384 x 512 29.1 -> 27.3 us, twelve to 32 of
// 8192 x 128 33.9 -> 31.1); a seventeenth warp costs registers, which 16 queries and 256 dimensions do not have (24 queries to 64 of 2000 x 256 36.7 -> 38.9)
template <int NQ, int UNITS> constexpr int MR_HELPERS = NQ * UNITS > 16 && NQ == 16 ? 1 : 2;
template <int NQ, int UNITS> constexpr int MR_THREADS = (7 + MR_HELPERS<NQ, UNITS> + 4 * MR_GROUPS<NQ, UNITS>) * 32;

// whether all 128 threads of a group of the softmax say so
__device__ __forceinline__ bool all_softmax(bool ok, int barrier)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)ok), "r"(barrier) : "memory");
    return r != 0;
}

// How a block's shared and tensor memory are laid out (the host's as well: it sizes them).
struct MapRows {
    int nby, nb;                              // blocks of 128 dimensions: of the bank, of the images
    int yslots, vslots;                       // of the bank, of values of their own
    int words;                                // words of scales of a point of the bank
    uint32_t x, p, scales, small;             // offsets: queries, weights (two buffers), scales (MR_AHEAD tiles', then the queries'), the rest
    uint32_t bytes, columns;
};
template <int NQ>
__host__ __device__ inline MapRows map_rows_layout(int d, int nb, int yslots, int vslots)
{
    MapRows L;
    L.nby = (d + 127) / 128;
    L.nb = nb;
    L.yslots = yslots;
    L.vslots = vslots;
    L.words = (L.nby + 3) / 4;
    L.x = (uint32_t)(yslots + vslots) * MR_SLOT;
    L.p = L.x + (uint32_t)(L.nby * MR_ROWS<NQ>) * 128;
    L.scales = L.p + 2 * (uint32_t)(L.nb * 2 * NQ) * 128;
    L.small = L.scales + (MR_AHEAD + 1) * (uint32_t)L.words * 512;
    // terms, values' scales, maxima, factors, tops, sums, runs, largest products, lengths, barriers
    L.bytes = L.small + MR_AHEAD * (128 * 4 + 128 * 8 + MR_MAX_BLOCKS * 4 + 4 * NQ * 4) + 12 * NQ * 16 + 2 * 4 * NQ * 4 + 2 * NQ * 4 + 2 * 4 * (uint32_t)nb * NQ * 4 +
              NQ * 8 + 64 * 8 + 32;
    const uint32_t used = 2 * MR_SCOLS<NQ> + 2 * (uint32_t)(L.nb * 2 * NQ) + 12 * (uint32_t)L.words;
    L.columns = 32;
    while (L.columns < used) L.columns *= 2;
    return L;
}

// four queries' weights of target p as two e4m3 numbers each, into a block of 128 dimensions' operand (from the target's byte on)
template <int NQ> __device__ __forceinline__ void put_weights(unsigned char *block, int p, int q, float a0, float a1, float a2, float a3)
{
    const uint32_t lo = e4m3_two(a0, a1), hi = e4m3_two(a2, a3);
    const float2 bl = e4m3_pair(lo), bh = e4m3_pair(hi);
    const uint32_t lo2 = e4m3_two((a0 - bl.x) * 16.f, (a1 - bl.y) * 16.f), hi2 = e4m3_two((a2 - bh.x) * 16.f, (a3 - bh.y) * 16.f);
    auto put = [&](int r, uint32_t byte) { block[r * 128 + (((p >> 4) ^ (r & 7)) << 4)] = (unsigned char)byte; };
    put(q, lo); put(q + 1, lo >> 8); put(q + 2, hi); put(q + 3, hi >> 8);
    put(NQ + q, lo2); put(NQ + q + 1, lo2 >> 8); put(NQ + q + 2, hi2); put(NQ + q + 3, hi2 >> 8);
}
// Values of a tile whose powers of two differ by more than MR_SPREAD: against the largest of them, weights of the others would leave the numbers' range, whatever
// little weight the largest has.  A query's weights times the powers are taken against the largest of these products then, 2^M of each 128
// dimensions (M - top, with weights against the tile's maximum), which takes that maximum, too, and a second barrier.  Calls, so that the usual way keeps its
// registers (one query to 8 banks of 16384 x 512: 27.2 us without this, 27.9 with calls, 29.1 in line; twelve to 32 of 8192 x 128 31.0, 31.1, 33.2).  Where
// every tile goes this way: twelve to 32 of 8192 x 128 with values of 64, 42; one to 8 of 16384 x 512 with values of 512, 40.7 for 38.0.
__device__ __forceinline__ float largest_of(const float *r, int stride) { return fmaxf(fmaxf(r[0], r[stride]), fmaxf(r[2 * stride], r[3 * stride])); }
__device__ __forceinline__ float less_top(float m, float top) { return m == -INFINITY ? 0.f : m - top; }
template <int NQ>
__device__ __noinline__ bool weights_apart(bool ok, const float (&arg)[NQ], const float4 *own, uint2 scales, float *reach, unsigned char *weights, int nb, int vblocks,
                                           int p, int nq, int barrier)
{
    const int lane = p & 31, part = p >> 5;
    auto power = [&](int u) { return (int)(((u < 4 ? scales.x : scales.y) >> (8 * (u & 3))) & 255u); };
    for (int u = 0; u < nb; ++u) {
        const float e = power(u) == 255 ? -INFINITY : (float)(power(u) - 127);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const float m = warp_max(arg[q] + e);
            if (lane == q) reach[(part * vblocks + u) * NQ + q] = m;
        }
    }
    if (!all_softmax(ok, barrier)) return false;
    for (int u = 0; u < nb; ++u) {
        const float e = power(u) == 255 ? __uint_as_float(0x7fffffffu) : (float)(power(u) - 119);              // (256 times)
#pragma unroll
        for (int q = 0; q < NQ; q += 4) {
            if (q >= nq) break;
            float a[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const float top = own[q + h].x;
                a[h] = arg[q + h] == -INFINITY ? 0.f : ex2_fast((arg[q + h] - top) + (e - less_top(largest_of(reach + u * NQ + q + h, vblocks * NQ), top)));
            }
            put_weights<NQ>(weights + u * (2 * NQ) * 128, p, q, a[0], a[1], a[2], a[3]);
        }
    }
    return true;
}
// ... and the tile's images, back to the weights' reference, in their place in tensor memory
template <int NQ>
__device__ __noinline__ void images_apart(uint32_t at, const float *reach, const float *maxima, int nb, int vblocks, int lane)
{
    for (int u = 0; u < nb; ++u) {
        float unit = 0.f;                                                            // of the query that is the lane's number
        if (lane < NQ) {
            const float top = largest_of(maxima + lane, NQ);
            unit = ex2_fast(less_top(largest_of(reach + u * NQ + lane, vblocks * NQ), top == -INFINITY ? 0.f : top));
        }
        uint32_t r[2 * NQ];
        if constexpr (NQ == 8) {
            tc_ld16_issue(at + u * 2 * NQ, r);
            tc_ld16_wait(r);
        } else {
            tc_ld32_issue(at + u * 2 * NQ, r);
            tc_ld_wait(r);
        }
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const float f = __shfl_sync(0xffffffffu, unit, q);
            r[q] = __float_as_uint(__uint_as_float(r[q]) * f);
            r[NQ + q] = __float_as_uint(__uint_as_float(r[NQ + q]) * f);
        }
        if constexpr (NQ == 8) tc_st16_issue(at + u * 2 * NQ, r);
        else tc_st32_issue(at + u * 2 * NQ, r);
    }
    tc_st_wait();
}

template <int NQ, int UNITS>
__global__ void __launch_bounds__(MR_THREADS<NQ, UNITS>) map_rows_kernel(const __grid_constant__ CUtensorMap tmy, const __grid_constant__ CUtensorMap tmv,
                                                              const __grid_constant__ Map P, const int yslots, const int vslots, const int vblocks)
{
    constexpr int ROWS = MR_ROWS<NQ>, SCOLS = MR_SCOLS<NQ>, GROUPS = MR_GROUPS<NQ, UNITS>;
    extern __shared__ __align__(1024) unsigned char smem[];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");               // (the parts' join waits for all of this grid's writes itself)
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // (values deeper than what a block has room for: further blocks, which form the scores again)
    const int qgroups = (P.n + NQ - 1) / NQ, z = blockIdx.x / qgroups, v0 = z * vblocks;
    const int split = blockIdx.y, q0 = (blockIdx.x - z * qgroups) * NQ, w = blockIdx.z, nq = min(NQ, P.n - q0);
    const MapRows L = map_rows_layout<NQ>(P.d, vblocks, yslots, vslots);
    const int nby = L.nby, nb = min(vblocks, (P.dv + 127) / 128 - v0);
    const uint32_t base = smem_u32(smem);
    float *terms = reinterpret_cast<float *>(smem + L.small);                        // [MR_AHEAD][128]
    uint2 *vscales = reinterpret_cast<uint2 *>(terms + MR_AHEAD * 128);              // [MR_AHEAD][128]
    float *maxima = reinterpret_cast<float *>(vscales + MR_AHEAD * 128);             // [MR_AHEAD][4][NQ]
    float4 *factors = reinterpret_cast<float4 *>(maxima + MR_AHEAD * 4 * NQ);        // [12][NQ]: each warp's own
    uint32_t *tops = reinterpret_cast<uint32_t *>(factors + 12 * NQ);                // [MR_AHEAD][8]
    float *sums = reinterpret_cast<float *>(tops + MR_AHEAD * MR_MAX_BLOCKS);        // [2][4][NQ]
    float *runs = sums + 8 * NQ;                                                     // [2][NQ]
    float *reach = runs + 2 * NQ;                                                    // [2][4][vblocks][NQ]
    double *lengths2 = reinterpret_cast<double *>(reach + 8 * vblocks * NQ);         // [NQ]
    unsigned long long *bars = reinterpret_cast<unsigned long long *>(lengths2 + NQ);
    uint32_t *holder = reinterpret_cast<uint32_t *>(bars + 64);
    int *abort_flag = reinterpret_cast<int *>(holder + 1);
    uint32_t *spread = reinterpret_cast<uint32_t *>(abort_flag + 1);                 // [MR_AHEAD]
    volatile int *ab = abort_flag;
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    constexpr int FULL = 0, EMPTY = MR_MAX_SLOTS, CFULL = 2 * MR_MAX_SLOTS, CEMPTY = CFULL + MR_AHEAD, SFULL = CEMPTY + MR_AHEAD, PFULL = SFULL + 2, DFULL = PFULL + 2,
                  DFREE = DFULL + 2, SFREE = DFREE + 2, MFULL = SFREE + 2, LAST = MFULL + MR_AHEAD;
    static_assert(LAST + 1 < 64, "barriers");

    const int len = map_length(P, w), tiles = (len + MR_T - 1) / MR_T;
    const int t0 = (int)((long long)tiles * split / P.splits), nt = (int)((long long)tiles * (split + 1) / P.splits) - t0;
    if (tid == 0) {
        for (int s = 0; s < yslots + vslots; ++s) { mbar_init(bar(FULL + s), 1); mbar_init(bar(EMPTY + s), 1); }
        for (int c = 0; c < MR_AHEAD; ++c) { mbar_init(bar(CFULL + c), 1); mbar_init(bar(CEMPTY + c), 8); mbar_init(bar(MFULL + c), 4); }
        for (int b = 0; b < 2; ++b) {
            mbar_init(bar(SFULL + b), 1);
            mbar_init(bar(PFULL + b), 4);
            mbar_init(bar(DFULL + b), 1);
            mbar_init(bar(DFREE + b), 4);
            mbar_init(bar(SFREE + b), 4);
        }
        mbar_init(bar(LAST), 1);
        mbar_init(bar(LAST + 1), 1);
        *abort_flag = (base & 1023u) ? 1 : 0;                                        // (the swizzle counts from 1024-byte boundaries)
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(holder)), "r"(L.columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const double k = map_scale(P, w);
    // Loads and targets' terms start at once; the others make the queries ready first.  What no query and no live weight fills stays zero: rows of
    // queries that are not there, their weights, the queries' unused scales
    constexpr int READY = 9 * 32;
    const int member = warp == 9 ? 8 : warp;
    if (warp < 8 || warp == 9) {
        for (uint32_t i = L.x / 16 + member * 32 + lane; i < L.scales / 16; i += READY) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0u, 0u, 0u, 0u);
        for (uint32_t i = (L.scales + MR_AHEAD * L.words * 512) / 16 + member * 32 + lane; i < L.small / 16; i += READY) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("bar.sync 3, %0;" ::"n"(READY) : "memory");
    }
    // the queries, a warp to each: blocks' powers of two, three numbers of a value, the squared length
    for (int q = member; q < nq && (warp < 8 || warp == 9); q += READY / 32) {
        const uint16_t *x = P.x + ((size_t)w * P.n + q0 + q) * P.d;
        double xx = 0.0;
        bool bad = false;
#pragma unroll 4
        for (int b = 0; b < nby; ++b) {
            float v[4], top = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int dim = 128 * b + 4 * lane + e;
                v[e] = dim < P.d ? __uint_as_float((uint32_t)x[dim] << 16) : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                bad |= !(fabsf(v[e]) <= 3.402823466e38f);
                top = fmaxf(top, fabsf(v[e]));
                xx += (double)v[e] * (double)v[e];
            }
            top = warp_max(top);
            int ex = CLOUD8_MIN_E;
            if (top > 0.f && top <= 3.402823466e38f) {
                ex = max(exponent_of(top) - 8, CLOUD8_MIN_E);
                if (top > 448.f * power_of_two(ex)) ++ex;
            }
            const float inv = power_of_two(-ex);
            float u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = v[e] * inv;
#pragma unroll
            for (int part = 0; part < 3; ++part) {
                const int r = part * NQ + q;
                const uint32_t lo = e4m3_two(u[0], u[1]), hi = e4m3_two(u[2], u[3]);
                *reinterpret_cast<uint32_t *>(smem + L.x + (b * ROWS + r) * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4) = lo | hi << 16;
                const float2 a = e4m3_pair(lo), c = e4m3_pair(hi);
                u[0] = (u[0] - a.x) * 16.f;
                u[1] = (u[1] - a.y) * 16.f;
                u[2] = (u[2] - c.x) * 16.f;
                u[3] = (u[3] - c.y) * 16.f;
                if (lane == 0) smem[L.scales + (MR_AHEAD * L.words + b / 4) * 512 + (r & 31) * 16 + (r >> 5) * 4 + (b & 3)] = (uint8_t)(ex - 4 * part + 127);
            }
        }
        bad = __any_sync(0xffffffffu, bad);
        __syncwarp();
        // (a query that is not finite: scales that are NaN)
        if (bad && lane < nby)
            for (int part = 0; part < 3; ++part) {
                const int r = part * NQ + q;
                smem[L.scales + (MR_AHEAD * L.words + lane / 4) * 512 + (r & 31) * 16 + (r >> 5) * 4 + (lane & 3)] = 255;
            }
#pragma unroll
        for (int off = 16; off; off /= 2) xx += __shfl_xor_sync(0xffffffffu, xx, off);
        if (lane == 0) lengths2[q] = xx;
        __syncwarp();
    }
    if (warp < 8 || warp == 9) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("bar.sync 3, %0;" ::"n"(READY) : "memory");
    }
    const uint32_t tmem = *holder;
    // tensor memory: scores (two buffers), images (two), the bank's scales (two), the queries'
    const uint32_t tD = tmem + 2 * SCOLS, dcols = (uint32_t)(vblocks * 2 * NQ), tA = tD + 2 * dcols, tB = tA + 8 * L.words;
    const bool starts = *ab == 0;
    auto there = [&](uint32_t a, uint32_t parity) {
        uint32_t r;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(r) : "r"(a), "r"(parity) : "memory");
        return r != 0;
    };
    // a tile's slots of a ring
    auto filled = [&](int first, int slots, int s, uint32_t ph, int count) {
        for (int c = 0; c < count; ++c) {
            if (!mbar_wait(bar(FULL + first + s), ph, ab)) return false;
            if (++s == slots) { s = 0; ph ^= 1u; }
        }
        return true;
    };
    // a query's largest exponent and the sum against it, of all groups
    auto total_of = [&](int q, float &top) {
        const float one = (sums[q] + sums[NQ + q]) + (sums[2 * NQ + q] + sums[3 * NQ + q]);
        top = runs[q];
        if constexpr (GROUPS == 1) return one;
        const float *more = sums + 4 * NQ;
        const float other = runs[NQ + q], two = (more[q] + more[NQ + q]) + (more[2 * NQ + q] + more[3 * NQ + q]);
        top = fmaxf(top, other);
        const float ref = top == -INFINITY ? 0.f : top;
        return one * ex2_fast(runs[q] - ref) + two * ex2_fast(other - ref);
    };
    // what a warp has issued is over before tensor memory is given back
    auto finish = [&](int barrier) {
        if (elected()) {
            tc_commit(bar(barrier));
            int unused = 0;
            mbar_wait(bar(barrier), 0, &unused);
        }
        __syncwarp();
    };

    constexpr int HELPERS = MR_HELPERS<NQ, UNITS>, SECOND = 8 + 4 * GROUPS;           // SECOND: the second of them, the last warp
    if (warp < 4 || (warp >= 12 && warp < SECOND)) {
        // ---- softmax: a thread to a target, which is a lane of tensor memory
        const int group = warp >> 3, part = warp & 3, p = part * 32 + lane;          // every other tile's
        const uint32_t lanes = (uint32_t)(part * 32) << 16;
        const float kx = (float)(2.0 * k);
        float4 *own = factors + (4 * group + part) * NQ;
        float run = -INFINITY, sum[NQ];                                              // run: of the query that is the lane's number
#pragma unroll
        for (int q = 0; q < NQ; ++q) sum[q] = 0.f;
        bool ok = starts;
        for (int t = group; t < nt && starts; t += GROUPS) {
            const int b = t & 1;
            const uint32_t ph = (uint32_t)(t >> 1) & 1u;
            const int c4 = t % MR_AHEAD;
            ok = ok && mbar_wait(bar(CFULL + c4), (uint32_t)(t / MR_AHEAD) & 1u, ab) && mbar_wait(bar(SFULL + b), ph, ab);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            const float term = terms[128 * c4 + p];
            const uint2 sv = vscales[128 * c4 + p];
            const bool masked = term == -INFINITY;
            // 256 times the values' powers of two, less the tile's largest (0: below fp32's), or NaN; masked targets have weights of zero
            float scale[UNITS];
            bool far = false;
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int e = (int)(((u < 4 ? sv.x : sv.y) >> (8 * (u & 3))) & 255u), x = e - (int)tops[c4 * MR_MAX_BLOCKS + u] + 135;
                scale[u] = __uint_as_float(e == 255 ? 0x7fffffffu : x > 0 ? (uint32_t)x << 23 : 0u);
                far |= x < 135 - MR_SPREAD;
            }
            far = __any_sync(0xffffffffu, far && !masked);
            float arg[NQ];
            if (ok) {
                uint32_t r[MR_SCOLS<NQ>];
                uint32_t (&r0)[32] = *reinterpret_cast<uint32_t (*)[32]>(r);
                tc_ld32_issue(tmem + lanes + SCOLS * b, r0);
                tc_ld_wait(r0);
                if constexpr (NQ == 16) {
                    uint32_t (&r1)[16] = *reinterpret_cast<uint32_t (*)[16]>(r + 32);
                    tc_ld16_issue(tmem + lanes + SCOLS * b + 32, r1);
                    tc_ld16_wait(r1);
                }
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const float s = __uint_as_float(r[q]) + (__uint_as_float(r[NQ + q]) + __uint_as_float(r[2 * NQ + q]));
                    arg[q] = masked ? -INFINITY : fmaf(s, kx, term);
                }
            } else
#pragma unroll
                for (int q = 0; q < NQ; ++q) arg[q] = 0.f;
            // (queries that are not there, to a whole four, have scores of zero: what becomes of them is not looked at)
#pragma unroll
            for (int q = 0; q < NQ; q += 4)
                if (q < nq) {
                    const float4 m = make_float4(warp_max(arg[q]), warp_max(arg[q + 1]), warp_max(arg[q + 2]), warp_max(arg[q + 3]));
                    if (lane == 0) *reinterpret_cast<float4 *>(maxima + (4 * c4 + part) * NQ + q) = m;
                }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(SFREE + b));                               // (the scores are in registers)
            // the weights of the tile before the last have been used; of the maxima there are as many as tiles ahead
            ok = ok && mbar_wait(bar(DFULL + b), ph ^ 1u, ab);
            if (far && lane == 0) spread[c4] = 1u;
            ok = all_softmax(ok, group ? 4 : 1);
            if (!ok) break;
            // a lane to a query: the tile's largest exponent, and what the sums so far and the tile's are multiplied by
            if (lane < NQ) {
                const float *mp = maxima + 4 * c4 * NQ + lane;
                const float top = fmaxf(fmaxf(mp[0], mp[NQ]), fmaxf(mp[2 * NQ], mp[3 * NQ])), now = fmaxf(run, top), ref = now == -INFINITY ? 0.f : now;
                own[lane] = make_float4(top == -INFINITY ? 0.f : top, ex2_fast(run - ref), ex2_fast(top - ref), 0.f);
                run = now;
            }
            __syncwarp();
            unsigned char *weights = smem + L.p + b * (vblocks * 2 * NQ) * 128 + (p & 15);
#pragma unroll
            for (int q = 0; q < NQ; q += 4) {
                if (q >= nq) break;
                float e[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const float4 f = own[q + h];
                    // (tile's maximum plus infinity: the exponential is NaN, and so is what follows from it)
                    e[h] = ex2_fast(arg[q + h] - f.x);
                    sum[q + h] = fmaf(sum[q + h], f.y, e[h] * f.z);
                }
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    if (u >= nb) break;
                    put_weights<NQ>(weights + u * (2 * NQ) * 128, p, q, masked ? 0.f : e[0] * scale[u], masked ? 0.f : e[1] * scale[u], masked ? 0.f : e[2] * scale[u],
                                    masked ? 0.f : e[3] * scale[u]);
                }
            }
            if (spread[c4]) {
                float again[NQ];
#pragma unroll
                for (int q = 0; q < NQ; ++q) again[q] = arg[q];
                // (the products of the tile before the last have been used, by the images as well)
                ok = mbar_wait(bar(DFREE + b), ph ^ 1u, ab);
                ok = weights_apart<NQ>(ok, again, own, sv, reach + b * 4 * vblocks * NQ, weights, nb, vblocks, p, nq, group ? 4 : 1);
                if (!ok) break;
                if (p < MR_MAX_BLOCKS) tops[c4 * MR_MAX_BLOCKS + p] = 127u;           // (what the images are multiplied by: they are whole as they are)
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            tc_fence_before();
            __syncwarp();
            if (lane == 0) { mbar_arrive(bar(PFULL + b)); mbar_arrive(bar(MFULL + c4)); mbar_arrive(bar(CEMPTY + c4)); }
        }
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            if (q >= nq) break;
            float s = ok ? sum[q] : __uint_as_float(0x7fffffffu);
#pragma unroll
            for (int off = 16; off; off /= 2) s += __shfl_xor_sync(0xffffffffu, s, off);
            if (lane == 0) sums[(4 * group + part) * NQ + q] = s;
        }
        if (p < NQ) runs[group * NQ + p] = run;
        asm volatile("bar.sync 2, %0;" ::"n"(128 + 128 * GROUPS) : "memory");
        if (tid < nq) {
            const size_t r = (size_t)w * P.n + q0 + tid;
            float top;
            const float total = total_of(tid, top);
            if (z == 0 && P.splits > 1) reinterpret_cast<float2 *>(P.part_ml)[r * P.splits + split] = make_float2(top, total);
            if (z == 0 && P.splits == 1 && P.lse) P.lse[r] = map_lse(top, total, k, lengths2[tid]);
        }
    } else if (warp < 8) {
        // ---- images: a thread to a dimension of every block
        const uint32_t lanes = (uint32_t)((warp - 4) * 32) << 16;
        float4 *own = factors + (4 + warp) * NQ;
        float out[UNITS][NQ], run = -INFINITY;
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int q = 0; q < NQ; ++q) out[u][q] = 0.f;
        bool ok = starts;
        for (int t = 0; t < nt && ok; ++t) {
            const int b = t & 1;
            const uint32_t ph = (uint32_t)(t >> 1) & 1u;
            // (the maxima by a barrier of their own, of which there are as many as tiles ahead: that of the weights may be a phase further by now, and a wait
            // for a phase that is followed by another complete one is over only with the one after that)
            ok = mbar_wait(bar(MFULL + t % MR_AHEAD), (uint32_t)(t / MR_AHEAD) & 1u, ab) && mbar_wait(bar(DFULL + b), ph, ab);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const bool apart = spread[t % MR_AHEAD] != 0;
            if (apart) images_apart<NQ>(tD + lanes + b * dcols, reach + b * 4 * vblocks * NQ, maxima + 4 * (t % MR_AHEAD) * NQ, nb, vblocks, lane);
            // what the images so far and the tile's are multiplied by
            __syncwarp();
            if (lane < NQ) {
                const float *mp = maxima + 4 * (t % MR_AHEAD) * NQ + lane;
                const float top = fmaxf(fmaxf(mp[0], mp[NQ]), fmaxf(mp[2 * NQ], mp[3 * NQ])), now = fmaxf(run, top), ref = now == -INFINITY ? 0.f : now;
                reinterpret_cast<float2 *>(own)[lane] = make_float2(ex2_fast(run - ref), ex2_fast(top - ref) * 0.00390625f);
                run = now;
            }
            __syncwarp();
            float before[NQ], of_tile[NQ];
#pragma unroll
            for (int q = 0; q < NQ; q += 2) {
                const float4 f = own[q / 2];
                before[q] = f.x;
                of_tile[q] = f.y;
                before[q + 1] = f.z;
                of_tile[q + 1] = f.w;
            }
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                if (u >= nb) break;
                const float unit = e8m0_value(tops[t % MR_AHEAD * MR_MAX_BLOCKS + u]);
                uint32_t r[2 * NQ];
                if constexpr (NQ == 8) {
                    tc_ld16_issue(tD + lanes + b * dcols + u * 2 * NQ, r);
                    tc_ld16_wait(r);
                } else {
                    tc_ld32_issue(tD + lanes + b * dcols + u * 2 * NQ, r);
                    tc_ld_wait(r);
                }
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const float v = fmaf(__uint_as_float(r[NQ + q]), 0.0625f, __uint_as_float(r[q])) * unit;
                    out[u][q] = fmaf(out[u][q], before[q], v * of_tile[q]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) { mbar_arrive(bar(DFREE + b)); mbar_arrive(bar(CEMPTY + t % MR_AHEAD)); }
        }
        asm volatile("bar.sync 2, %0;" ::"n"(128 + 128 * GROUPS) : "memory");
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            if (q >= nq) break;
            const size_t r = (size_t)w * P.n + q0 + q;
            // (of parts, the join divides)
            float inv = 1.f, top;
            if (P.splits == 1) {
                const float total = total_of(q, top);
                inv = total == 0.f ? 0.f : 1.f / total;
            }
            if (!ok) inv = __uint_as_float(0x7fffffffu);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int dim = 128 * (v0 + u) + tid - 128;
                if (u >= nb || dim >= P.dv) continue;
                if (P.splits > 1) P.part_out[(r * P.splits + split) * P.dv + dim] = out[u][q] * inv;
                else P.out[r * P.dv + dim] = (uint16_t)bf16_pair(out[u][q] * inv, 0.f);
            }
        }
    } else if (warp == 8) {
        // ---- loads: of the bank and of values of their own, whichever has a slot
        if (lane == 0) {
            bool ok = starts;
            struct Ring {
                int slot, block, tile, issued;
                uint32_t ph;
            } ring[2] = {{0, 0, 0, 0, 0u}, {0, 0, vslots ? 0 : nt, 0, 0u}};
            auto move = [&](Ring &r, bool value) {
                const int first = value ? yslots : 0, slots = value ? vslots : yslots;
                if (r.tile >= nt || !there(bar(EMPTY + first + r.slot), r.ph ^ 1u)) return false;
                const uint32_t full = bar(FULL + first + r.slot), dst = base + (first + r.slot) * MR_SLOT;
                mbar_expect_tx(full, MR_SLOT);
                if (value) tma_points(dst, &tmv, (v0 + r.block) * 128, (t0 + r.tile) * MR_T, w, full);
                else tma_points(dst, &tmy, r.block * 128, (t0 + r.tile) * MR_T, w, full);
                ++r.issued;
                if (++r.block == (value ? nb : nby)) { r.block = 0; ++r.tile; }
                if (++r.slot == slots) { r.slot = 0; r.ph ^= 1u; }
                return true;
            };
            long long since = clock64();
            while (ok && (ring[0].tile < nt || ring[1].tile < nt)) {
                const bool a = move(ring[0], false), b = move(ring[1], true);
                if (a || b) since = clock64();
                else if (*ab || clock64() - since > TC_WAIT_CLOCKS) {
                    *abort_flag = 1;
                    ok = false;
                }
            }
            // nothing may land in shared memory after the block has gone: the last load of every slot, with a bound of its own
            int unused = 0;
            for (int q = max(0, ring[0].issued - yslots); q < ring[0].issued; ++q) mbar_wait(bar(FULL + q % yslots), (uint32_t)(q / yslots) & 1u, &unused);
            for (int q = max(0, ring[1].issued - vslots); q < ring[1].issued; ++q)
                mbar_wait(bar(FULL + yslots + q % vslots), (uint32_t)(q / vslots) & 1u, &unused);
        }
    } else if (warp == 9) {
        // ---- scores: the whole warp walks through the tiles, so that descriptors are uniform; one thread issues.  (A wait, and what follows it, takes as
        // long as sixteen instructions: a tile's slots are waited for first, then all is issued.)
        constexpr uint32_t shape = ((uint32_t)(ROWS >> 3) << 17) | ((uint32_t)(128 >> 4) << 24) | 1u << 23;            // e4m3, e4m3, scales e8m0
        const uint64_t y0 = tc_desc(base), x0 = tc_desc(base + L.x);
        const int steps_last = (P.y.cb - 128 * (nby - 1)) / 32;
        int slot0 = 0;
        uint32_t ph = 0;
        bool ok = starts;
        for (int t = 0; t < nt && ok; ++t) {
            const int b = t & 1;
            ok = mbar_wait(bar(CFULL + t % MR_AHEAD), (uint32_t)(t / MR_AHEAD) & 1u, ab) && mbar_wait(bar(SFREE + b), ((uint32_t)(t >> 1) & 1u) ^ 1u, ab) &&
                 filled(0, yslots, slot0, ph, nby);
            if (!(ok = __all_sync(0xffffffffu, ok))) break;
            tc_fence_after();
            if (elected()) {
                for (int a = 0; a < L.words; ++a) {
                    scales_in(tA + (b * L.words + a) * 4, base + L.scales + (t % MR_AHEAD * L.words + a) * 512);
                    if (t == 0) scales_in(tB + a * 4, base + L.scales + (MR_AHEAD * L.words + a) * 512);
                }
                const uint32_t acc = tmem + SCOLS * b;
                int slot = slot0;
                for (int c = 0; c < nby; ++c) {
                    const uint64_t yd = y0 + (uint64_t)(slot * (int)(MR_SLOT >> 4)), xd = x0 + (uint64_t)(c * (ROWS * 128 >> 4));
                    const uint32_t part = (uint32_t)(c & 3), idesc = shape | part << 29 | part << 4;
                    const uint32_t sfa = tA + (b * L.words + c / 4) * 4, sfb = tB + (c / 4) * 4;
                    mma_scaled(acc, yd, xd, idesc, sfa, sfb, c ? 1u : 0u);
                    if (c < nby - 1 || steps_last == 4) {
#pragma unroll
                        for (int q = 1; q < 4; ++q) mma_scaled(acc, yd + 2 * q, xd + 2 * q, idesc, sfa, sfb, 1u);
                    } else
                        for (int q = 1; q < steps_last; ++q) mma_scaled(acc, yd + 2 * q, xd + 2 * q, idesc, sfa, sfb, 1u);
                    if (vslots) tc_commit(bar(EMPTY + slot));
                    if (++slot == yslots) slot = 0;
                }
                tc_commit(bar(SFULL + b));
            }
            __syncwarp();
            slot0 += nby;
            if (slot0 >= yslots) { slot0 -= yslots; ph ^= 1u; }
        }
        finish(LAST);
    } else if (warp == 11) {
        // ---- images
        constexpr uint32_t shape = (1u << 4) | 1u << 15 | ((uint32_t)(2 * NQ >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);   // D fp32, A M-major
        const uint64_t y0 = tc_desc(base), p0 = tc_desc(base + L.p);
        const int first = vslots ? yslots : 0, slots = vslots ? vslots : yslots;
        int slot0 = 0;
        uint32_t ph = 0;
        bool ok = starts;
        for (int t = 0; t < nt && ok; ++t) {
            const int b = t & 1;
            // (values that are the bank are there: the weights are made of its scores.  Waited for all the same, which orders the reads.)
            // The weights, which come last, are waited for last.
            ok = mbar_wait(bar(DFREE + b), ((uint32_t)(t >> 1) & 1u) ^ 1u, ab) && filled(first, slots, slot0, ph, nb) && mbar_wait(bar(PFULL + b), (uint32_t)(t >> 1) & 1u, ab);
            if (!(ok = __all_sync(0xffffffffu, ok))) break;
            tc_fence_after();
            if (elected()) {
                int slot = slot0;
                for (int c = 0; c < nb; ++c) {
                    const uint64_t vd = y0 + (uint64_t)((first + slot) * (int)(MR_SLOT >> 4)), pd = p0 + (uint64_t)((b * vblocks + c) * (2 * NQ * 128 >> 4));
                    const uint32_t acc = tD + b * dcols + c * 2 * NQ;
#pragma unroll
                    for (int q = 0; q < 4; ++q) mma_codes(acc, vd + q * (4096 >> 4), pd + 2 * q, shape, q ? 1u : 0u);
                    tc_commit(bar(EMPTY + first + slot));
                    if (++slot == slots) slot = 0;
                }
                tc_commit(bar(DFULL + b));
            }
            __syncwarp();
            slot0 += nb;
            if (slot0 >= slots) { slot0 -= slots; ph ^= 1u; }
        }
        finish(LAST + 1);
    } else {
        // ---- targets' scales and terms, a lane to every 32nd target of a tile; two tiles' of a warp on their way from memory, all of a tile's
        // loads at once
        struct Raw {
            double g[4];
            float norm[4];
            uint32_t y0[4], y1[4], v0[4], v1[4];
        };
        const int words_v = P.v.sb / 4, word = v0 / 4, shift = 8 * (v0 & 3);       // scales from the first block of this block's dimensions on
        auto fetch = [&](int t, Raw &r) {
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const size_t at = (size_t)w * P.m + min((t0 + t) * MR_T + lane + 32 * a, len - 1);
                const uint32_t *sy = reinterpret_cast<const uint32_t *>(P.y.scales + at * P.y.sb), *sv = reinterpret_cast<const uint32_t *>(P.v.scales + at * P.v.sb) + word;
                r.g[a] = P.g ? P.g[at] : 0.0;
                r.norm[a] = P.y.norms[at];
                r.y0[a] = sy[0];
                r.y1[a] = L.words > 1 ? sy[1] : 0u;
                r.v0[a] = P.own_values ? sv[0] : 0u;
                r.v1[a] = P.own_values && word + 1 < words_v ? sv[1] : 0u;
            }
        };
        bool ok = starts;
        auto give = [&](int t, Raw &r) {
            const int b = t % MR_AHEAD;
            ok = __all_sync(0xffffffffu, mbar_wait(bar(CEMPTY + b), ((uint32_t)(t / MR_AHEAD) & 1u) ^ 1u, ab));
            if (!ok) return;
            uint4 *dst = reinterpret_cast<uint4 *>(smem + L.scales + b * L.words * 512) + lane;
            dst[0] = make_uint4(r.y0[0], r.y0[1], r.y0[2], r.y0[3]);
            if (L.words > 1) dst[32] = make_uint4(r.y1[0], r.y1[1], r.y1[2], r.y1[3]);
            bool masked[4];
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const int p = lane + 32 * a;
                const float term = (t0 + t) * MR_T + p < len ? map_term(k, r.g[a], r.norm[a]) : -INFINITY;
                masked[a] = term == -INFINITY;
                if (P.own_values) {
                    r.v0[a] = __funnelshift_r(r.v0[a], r.v1[a], shift);
                    r.v1[a] >>= shift;
                } else { r.v0[a] = r.y0[a]; r.v1[a] = r.y1[a]; }
                terms[128 * b + p] = term;
                vscales[128 * b + p] = make_uint2(r.v0[a], r.v1[a]);
            }
            // the values' largest power of two of the tile in each block (of targets that are masked or NaN: none)
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                uint32_t top = 0;
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const uint32_t e = ((u < 4 ? r.v0[a] : r.v1[a]) >> (8 * (u & 3))) & 255u;
                    top = max(top, masked[a] || e == 255u ? 0u : e);
                }
                top = __reduce_max_sync(0xffffffffu, top);
                if (lane == 0) tops[b * MR_MAX_BLOCKS + u] = top;
            }
            if (lane == 0) spread[b] = 0u;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(CFULL + b));
        };
        Raw one, two;
        const int turn = HELPERS == 2 && warp == SECOND;
        if (turn < nt) fetch(turn, one);
        if (turn + HELPERS < nt) fetch(turn + HELPERS, two);
        for (int t = turn; t < nt && ok; t += 2 * HELPERS) {
            give(t, one);
            if (t + 2 * HELPERS < nt) fetch(t + 2 * HELPERS, one);
            if (t + HELPERS >= nt || !ok) break;
            give(t + HELPERS, two);
            if (t + 3 * HELPERS < nt) fetch(t + 3 * HELPERS, two);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L.columns) : "memory");
}

// The parts of a query's image, added up: a block to 128 dimensions of a query, a warp to every eighth part, in an order that does not change.
__global__ void __launch_bounds__(256) map_join_kernel(const __grid_constant__ Map P)
{
    __shared__ float s_out[8][128], s_sum[8];
    __shared__ double s_xx[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, dim0 = blockIdx.y * 128;
    const long long r = blockIdx.x;
    const bool sums = P.lse && dim0 == 0;
    double xx = 0.0;
    if (sums)                                                                // (the query does not wait for the parts)
        for (int i = threadIdx.x; i < P.d; i += 256) {
            const double v = __uint_as_float((uint32_t)P.x[r * P.d + i] << 16);
            xx += v * v;
        }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float2 *ml = reinterpret_cast<const float2 *>(P.part_ml) + r * P.splits;
    float top = -INFINITY;
    for (int s = lane; s < P.splits; s += 32) top = fmaxf(top, ml[s].x);
#pragma unroll
    for (int off = 16; off; off /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = warp; s < P.splits; s += 8) {
        const float2 one = ml[s];
        const float f = ex2_fast(one.x - ref);
        const float *src = P.part_out + (r * P.splits + s) * P.dv + dim0 + lane;
        sum = fmaf(one.y, f, sum);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (dim0 + lane + 32 * e < P.dv) v[e] = fmaf(src[32 * e], f, v[e]);
    }
#pragma unroll
    for (int off = 16; off; off /= 2) xx += __shfl_xor_sync(0xffffffffu, xx, off);
#pragma unroll
    for (int e = 0; e < 4; ++e) s_out[warp][lane + 32 * e] = v[e];
    if (lane == 0) { s_sum[warp] = sum; s_xx[warp] = xx; }
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += s_sum[i];
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int dim = dim0 + threadIdx.x;
    if (threadIdx.x < 128 && dim < P.dv) {
        float o = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) o += s_out[i][threadIdx.x];
        P.out[r * P.dv + dim] = (uint16_t)bf16_pair(o * inv, 0.f);
    }
    if (sums && threadIdx.x == 0) {
        xx = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) xx += s_xx[i];
        P.lse[r] = map_lse(top, sum, map_scale(P, (int)(r / P.n)), xx);
    }
}

// Slots of a block, and the blocks of 128 dimensions of the values that it takes.
struct RowsShape {
    int nq, yslots, vslots, vblocks, chunks;
};
template <int NQ>
RowsShape rows_shape(int d, int dv, bool own, long long tiles)
{
    const int nby = (d + 127) / 128, nb = (dv + 127) / 128, most = NQ == 16 ? 2 : MR_MAX_BLOCKS;
    RowsShape r = {};
    r.nq = NQ;
    // (chunks of values of their own are of four blocks, a word of scales, or whole)
    r.vblocks = nb;
    const auto slots = [&](int room) {
        const MapRows L = map_rows_layout<NQ>(d, r.vblocks, 0, 0);
        return min(MR_MAX_SLOTS, (room - (int)L.bytes) / (int)MR_SLOT);
    };
    if (own && slots(MAP_TILES_SMEM) < nby + nb) r.vblocks = 4;
    if (own && slots(MAP_TILES_SMEM) < nby + r.vblocks) r.vblocks = 2;
    if (r.vblocks > most) r.vblocks = most;
    r.chunks = (nb + r.vblocks - 1) / r.vblocks;
    const int per_tile = nby + (own ? r.vblocks : 0);
    const long long all = min((long long)slots(MAP_TILES_SMEM), max(2LL, tiles) * per_tile);
    // shares of the slots in proportion, a tile's blocks at least
    r.vslots = own ? max(r.vblocks, min((int)all - nby, (int)(all * r.vblocks / per_tile))) : 0;
    r.yslots = (int)all - r.vslots;
    return r;
}
template <int NQ, int UNITS>
skb_status launch_rows(const CUtensorMap &ty, const CUtensorMap &tv, const Map &P, const RowsShape &r, cudaStream_t st)
{
    const MapRows L = map_rows_layout<NQ>(P.d, r.vblocks, r.yslots, r.vslots);
    cudaFuncSetAttribute(map_rows_kernel<NQ, UNITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L.bytes);
    map_rows_kernel<NQ, UNITS><<<dim3((P.n + NQ - 1) / NQ * r.chunks, P.splits, P.W), MR_THREADS<NQ, UNITS>, L.bytes, st>>>(ty, tv, P, r.yslots, r.vslots, r.vblocks);
    return op_launched("map");
}
skb_status launch_rows_by_depth(const CUtensorMap &ty, const CUtensorMap &tv, const Map &P, int nq, cudaStream_t st)
{
    const long long tiles = ((P.m + MR_T - 1) / MR_T + P.splits - 1) / P.splits;
    if (nq == 16) {
        const RowsShape r = rows_shape<16>(P.d, P.dv, P.own_values != 0, tiles);
        return r.vblocks <= 1 ? launch_rows<16, 1>(ty, tv, P, r, st) : launch_rows<16, 2>(ty, tv, P, r, st);
    }
    const RowsShape r = rows_shape<8>(P.d, P.dv, P.own_values != 0, tiles);
    if (r.vblocks <= 1) return launch_rows<8, 1>(ty, tv, P, r, st);
    if (r.vblocks <= 2) return launch_rows<8, 2>(ty, tv, P, r, st);
    if (r.vblocks <= 4) return launch_rows<8, 4>(ty, tv, P, r, st);
    return launch_rows<8, 8>(ty, tv, P, r, st);
}

// What a call is shared out by: the kernel, queries to a block of map_rows_kernel, parts of a lane's bank.  The first two go by the sizes alone, as a
// B200's SMs take them, so that the workspace does not depend on the device.
constexpr int MAP_SMS = 148;
// Queries up to which the tiles of 128 queries are too empty to be worth the staging (us, here / with tiles; W, m, d, dv):
//      queries                     16          32          33          48          64
//      8, 16384, 512            41 / 92     72 / 98     94 / 99     95 / 100   131 / 109
//      32, 8192, 128, 64        30 / 66     49 / 67     82 / 68     71 / 69     82 / 70
//      64, 1024, 512            24 / 46     46 / 46     65 / 46     67 / 46     89 / 46
//      64, 1024, 128            14 / 22     18 / 24     31 / 24     34 / 27     35 / 30
constexpr int MAP_ROWS_MAX = 32;
// ... and beyond them while an SM has no more than so many tiles, for one launch less (24, 333, 200, 96: 48 queries, three tiles of eight, 11 / 13; 77, three
// of sixteen, 15 / 13, with the host's time 20 / 23; 128, six, 28 / 13; 1, 2000, 64: 128 queries, two tiles, 11 / 15)
constexpr int MAP_ROWS_STEPS = 4;

const char *map_refused(int W, int n, int m, int d, int dv)
{
    if (W < 1 || n < 1 || m < 1 || d < 1) return "W, n, m and d must be >= 1";
    if (W > 65535 || n > 262143 || m > 262143) return "W at most 65535, n and m at most 262143";
    if (d > CLOUD8_MAX_D || dv > CLOUD8_MAX_D || dv < 0) return "d and dv must be at most 1024";
    return nullptr;
}
struct MapPlan {
    bool tiles;
    int nq, splits;
};
// enough parts to fill the device, of a few tiles at least
int map_splits(long long blocks, long long tiles, int sms)
{
    const long long s = min(sms / blocks, tiles / 2);
    return (int)(s < 1 ? 1 : s > 128 ? 128 : s);
}
long long rows_blocks(const RowsShape &r, int W, int n) { return (long long)W * ((n + r.nq - 1) / r.nq) * r.chunks; }
// Tiles that an SM gets through one after the other, and what they take, in halves of a tile of eight queries: a tile of sixteen takes half as long again, the
// join of parts as long as two
struct RowsCost {
    long long tiles, time;
};
RowsCost rows_cost(const RowsShape &r, int W, int n, long long tiles)
{
    const long long blocks = rows_blocks(r, W, n), splits = map_splits(blocks, tiles, MAP_SMS);
    const long long steps = (blocks * splits + MAP_SMS - 1) / MAP_SMS * ((tiles + splits - 1) / splits);
    return {steps, steps * (r.nq == 16 ? 3 : 2) + (splits > 1 ? 4 : 0)};
}
MapPlan map_plan(int W, int n, int m, int d, int dv, bool own_values, int sms)
{
    const long long tiles = (m + MR_T - 1) / MR_T;
    RowsShape r = rows_shape<8>(d, dv, own_values, tiles);
    // Images above 256 dimensions have eight: registers leave one group of warps to the softmax of sixteen, which takes twice as long.  (us, with eight / sixteen: 32 x
    // 8192 x 128 with values of 64, 12 queries 33 / 28, 32 queries 55 / 48; 64 x 1024 x 128, 16 queries 14 / 17, 32 queries 26 / 18; 24 x 333 x 200, 24
    // queries 11 / 15)
    if (n > 8 && dv <= 256) {
        const RowsShape r16 = rows_shape<16>(d, dv, own_values, tiles);
        if (r16.yslots >= (d + 127) / 128 && rows_cost(r16, W, n, tiles).time < rows_cost(r, W, n, tiles).time) r = r16;
    }
    MapPlan p;
    p.nq = r.nq;
    p.tiles = d <= MAP_TILES_MAX_D && n > MAP_ROWS_MAX && rows_cost(r, W, n, tiles).tiles > MAP_ROWS_STEPS;
    p.splits = map_splits(p.tiles ? (long long)W * (n > 128 ? (n + 255) / 256 * 2 : 1) * ((dv + 255) / 256) : rows_blocks(r, W, n), tiles, sms);
    return p;
}
size_t pad256(size_t b) { return (b + 255) / 256 * 256; }
size_t map_parts_bytes(int W, int n, int dv, int splits)
{
    return splits == 1 ? 0 : pad256((size_t)W * n * splits * 8) + pad256((size_t)W * n * splits * dv * 4);
}

}  // namespace
}  // namespace skb

using namespace skb;

// own_values: dv is that of a cloud of its own
static size_t map_workspace(int W, int n, int m, int d, int dv, bool own_values)
{
    // (what any device may split into: the workspace does not depend on the current one)
    const MapPlan p = map_plan(W, n, m, d, dv, own_values, MAP_MAX_SMS);
    return 256 + map_parts_bytes(W, n, dv, p.splits) + (p.tiles ? pad256(map_staged_bytes(W, n, m, d, dv, own_values, p.splits)) : 0);
}

extern "C" size_t sinkhorn_cloud8_map_workspace_bytes(int W, int n, int m, int d, int dv)
{
    return map_refused(W, n, m, d, dv) ? 0 : map_workspace(W, n, m, d, dv ? dv : d, dv != 0);
}

extern "C" skb_status sinkhorn_cloud8_map(const void *x, const void *y, const double *g, const float *eps, const void *v, const int *lengths, int W, int n, int m,
                                          int d, int dv, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!x || !y || !eps || !out || !workspace) return op_fail(SKB_ERR_NULL, "x, y, eps, out and workspace are required");
    if (const char *why = map_refused(W, n, m, d, v ? dv : d)) return op_fail(SKB_ERR_SHAPE, why);
    if (v && dv < 1) return op_fail(SKB_ERR_SHAPE, "values of their own have a depth dv >= 1");
    if (const char *why = cloud8_refused(W, m, d)) return op_fail(SKB_ERR_SHAPE, why);
    if ((uintptr_t)y % 256 || (uintptr_t)v % 256 || (uintptr_t)workspace % 256) return op_fail(SKB_ERR_WORKSPACE, "y, v and workspace must be 256-byte aligned");
    if ((uintptr_t)x % 2 || (uintptr_t)out % 2 || (uintptr_t)g % 8 || (uintptr_t)eps % 4 || (uintptr_t)lse % 4 || (uintptr_t)lengths % 4)
        return op_fail(SKB_ERR_WORKSPACE, "arrays must be aligned to their types");
    const int depth = v ? dv : d;
    if (workspace_bytes < map_workspace(W, n, m, d, depth, v != nullptr)) return op_fail(SKB_ERR_WORKSPACE, "workspace too small");
    // (a block's queries may be read after another block has written images)
    const uintptr_t x0 = (uintptr_t)x, out0 = (uintptr_t)out, queries = (uintptr_t)W * n;
    if (x0 < out0 + 2 * queries * depth && out0 < x0 + 2 * queries * d) return op_fail(SKB_ERR_VALUE, "images cannot take the place of the queries");
    int dev = 0, sms = 0;
    cudaGetDevice(&dev);
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return op_launched("device");
    Map P = {};
    P.x = (const uint16_t *)x;
    P.y = cloud8_view(y, (size_t)W * m, d);
    P.v = v ? cloud8_view(v, (size_t)W * m, dv) : P.y;
    P.g = g; P.eps = eps; P.lengths = lengths; P.out = (uint16_t *)out; P.lse = lse;
    P.W = W; P.n = n; P.m = m; P.d = d; P.dv = depth; P.own_values = v != nullptr;
    const MapPlan plan = map_plan(W, n, m, d, depth, v != nullptr, sms < MAP_MAX_SMS ? sms : MAP_MAX_SMS);
    P.splits = plan.splits;
    P.part_ml = (float *)workspace;
    P.part_out = (float *)((char *)workspace + pad256((size_t)W * n * P.splits * 8));
    void *room = (char *)workspace + map_parts_bytes(W, n, depth, P.splits);
    CUtensorMap ty, tv;
    if (!plan.tiles && (!points_map(&ty, P.y.codes, P.y.cb, m, W, MR_T) || !points_map(&tv, P.v.codes, P.v.cb, m, W, MR_T)))
        return op_fail(SKB_ERR_CUDA, "cuTensorMapEncodeTiled failed");
    const skb_status rc = plan.tiles ? launch_map_tiles(P, room, sms, (cudaStream_t)stream) : launch_rows_by_depth(ty, tv, P, plan.nq, (cudaStream_t)stream);
    if (rc != SKB_OK || P.splits == 1) return rc;
    // (it may start, and wait, before the parts are all there)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(W * n, (depth + 127) / 128);
    cfg.blockDim = dim3(256);
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, map_join_kernel, P);
    return op_launched("map");
}
