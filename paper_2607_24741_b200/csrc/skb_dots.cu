// Products of two clouds, out[t, i, j] = x_ti . y_tj in fp32: 4-bit clouds by the block-scaled matrix instructions
// (mx4: kind::mxf4, scales of 32 dimensions; nv4: kind::mxf4nvf4, scales of 16), 8-bit clouds by kind::mxf8f6f4 (a scale of 128 dimensions
// serves four instructions), bf16 clouds by kind::f16.
//
// The operands are small (a point of 512 dimensions in 4 bits is 272 bytes) and the result is not: 4 n m bytes a lane
// bound the kernel (64 lanes of 1024 x 1024: 268 MB, 41 us at the measured copy rate; the 69 GFLOP would take 11 us at
// four times the bf16 rate).  So the kernel is one persistent block an SM that always has a tile of results on its way out:
//   warp 0     loads, by TMA: chunks of 128 bytes a point (256 dimensions in 4 bits, 128 in 8, 64 in bf16), 128 points of x and of y,
//              128-byte swizzle; points and dimensions past the end arrive as zeros
//   warp 1     matrix instructions, one thread: four to a chunk into one of two accumulators of 128 x 128 in tensor memory
//   warps 2-5  block scales (all but bf16): from the points' rows into the order that the matrix unit wants, through
//              shared memory; they are a sixteenth of the codes and their rows too short for TMA.  Two warps to an operand, each
//              takes every other chunk, so that a chunk's load latency has two chunks' time
//   warps 6-13 results: tensor memory -> registers -> 32 x 32 boxes in shared memory -> TMA stores, which clip ragged edges.
//              Rows that are no whole number of 16 bytes are stored by the threads, a warp to a row
// Tiles are dealt out to the blocks in turn, columns fastest: what is written at a time lies together.  A range of tiles to a block
// with the rows' operand kept in shared memory reads half as much and takes longer (64 lanes of 1024 x 1024 x 512, mx4: 71 us,
// pairs of tiles with their rows kept 61, this 56; a fill of the same results 39).  In 8 bits the same results take 82 us: twice as much, 537 MB, goes from
// L2 to the SMs beside the 268 MB that are written (rows kept: 95; all scales of a tile loaded a tile ahead: the same).  Four warps for the results instead
// of eight: 73 us for 4 lanes of 4096 x 4096 x 512 in nv4, 68 so.
// In nv4 the points' powers of two multiply the results on their way out, which is exact.
// Accumulation is the matrix unit's fp32, which cuts off: measured with sums made for it, every product of an instruction (4-bit kinds: every
// block of a common scale) and the sum so far are cut at 2^-25 of the power of two of the largest of them, and the result to its 24
// bits.  Beside a sum that is there from the start 512 dimensions of bf16 can lose 127 units in its last place that way.  Draws
// have to know their products' errors, and larger ones leave more rows to be formed again: bf16 products are summed 64 dimensions at a time, and
// these sums added by the warps for the results, in fp32's rounding.  Every wait is bounded (skb_tmem.cuh): one that runs out ends all roles, and
// the tiles that were not finished are NaN.
#include <cuda.h>
#include <cuda_runtime.h>
#include <string>

#include "skb_cloud8.cuh"
#include "skb_operators.h"
#include "skb_tmem.cuh"

namespace skb {
namespace {

constexpr int DT_BM = 128, DT_BN = 128;
constexpr int DT_EPI = 8, DT_THREADS = (6 + DT_EPI) * 32, DT_STAGES = 4;
constexpr uint32_t DT_TILE = 128 * 128;                  // bytes: 128 points, 128 bytes of each
constexpr uint32_t DT_BOX = 32 * 32 * 4;                 // a box of results
// chunks of an accumulator (4-bit kinds have at most four, 8-bit clouds eight)
template <int KIND> constexpr int DT_PART = KIND == SKB_BF16 ? DOTS_BF16_PART / 64 : 8;
constexpr int DT_SF_COL = 2 * DT_BN, DT_SF_STRIDE = 32;  // tensor memory: accumulators, then the scales of each stage

struct Dots {
    const uint8_t *sx, *sy;                               // scales (all but bf16)
    const float *px, *py;                                 // points' powers of two (nv4)
    float *out;
    long long ldo, lane_out;                              // floats from row to row, from lane to lane
    int W, n, m, no, mo, row_bytes, sb;                   // no, mo: rows and columns of results; row_bytes: of a point's codes (or bf16 values)
    int tma_out;
};

template <int KIND>
__device__ __forceinline__ constexpr uint32_t dots_idesc()
{
    constexpr uint32_t shape = ((uint32_t)(DT_BN >> 3) << 17) | ((uint32_t)(DT_BM >> 4) << 24);
    if (KIND == SKB_BF16) return (1u << 4) | (1u << 7) | (1u << 10) | shape;             // D fp32, A and B bf16
    if (KIND == FMT_MX8) return shape | 1u << 23;                                        // A and B e4m3; scales e8m0
    return (1u << 7) | (1u << 10) | shape | (KIND == SKB_MX4 ? 1u << 23 : 0u);           // A and B e2m1; scales e8m0 or e4m3
}
template <int KIND>
__device__ __forceinline__ void dots_mma(uint32_t acc, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate)
{
    if constexpr (KIND == SKB_BF16) tc_mma(acc, a, b, idesc, accumulate);
    else if constexpr (KIND == SKB_MX4)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     ::"r"(acc), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb) : "memory");
    else if constexpr (KIND == FMT_MX8)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     ::"r"(acc), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     ::"r"(acc), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb) : "memory");
}
// 128 points' words of four scales, 512 bytes of shared memory, into four columns of tensor memory, the same for all four
// quarters of the lanes.  Rows of 16 bytes, eight to a group of 128 bytes, no swizzle.
__device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint32_t saddr)
{
    const uint64_t desc = (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(128u >> 4) << 32) | (1ull << 46);
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void tma_load_points(uint32_t dst, const CUtensorMap *tm, int byte, int point, int lane, uint32_t mbar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(byte), "r"(point), "r"(lane), "r"(mbar) : "memory");
}
__device__ __forceinline__ void tma_store_box(const CUtensorMap *tm, uint32_t src, int col, int row, int lane)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(reinterpret_cast<uint64_t>(tm)), "r"(col), "r"(row), "r"(lane), "r"(src) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

// A sum in units of two points' powers of two, rounded once.  It is 0 or between 2^-20 and 2^33, and powers within FAR_POINT of 1 can
// multiply it in any order; for others sum * a may be infinite, or have lost bits, where sum * a * b is neither.
constexpr float FAR_POINT = 1099511627776.f;             // 2^40
__device__ __forceinline__ bool far_point(float p) { return p > FAR_POINT || p < 1.f / FAR_POINT; }
__device__ __forceinline__ float times_points(float sum, float a, float b)
{
    if ((a > 1.f) != (b > 1.f)) return sum * (a * b);
    // both above 1: infinite at the first step is infinite in the end; both below: bits are lost at the first where the end is 0
    return sum * fmaxf(a, b) * fminf(a, b);
}

// A warp's 32 rows and 64 columns of a tile with points far from 1 (nv4), by way of one of its boxes.
__device__ __noinline__ void far_tile(const Dots &P, unsigned char *box, uint32_t src, bool ok, int w, int row0, int col0, float rp, const float *cps, int lane)
{
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
        const int col = col0 + 32 * h;
        if (col >= P.mo || row0 >= P.no) break;
        uint32_t r[32];
        tc_ld32_issue(src + 32 * h, r);
        tc_ld_wait(r);
        // (threads next to each other to banks next to each other: element q of row l at 32 l + (q + l) % 32)
#pragma unroll
        for (int q = 0; q < 32; ++q)
            reinterpret_cast<float *>(box)[32 * lane + ((q + lane) & 31)] = ok ? times_points(__uint_as_float(r[q]), rp, cps[32 * h + q]) : __uint_as_float(0x7fffffffu);
        __syncwarp();
        const int rows = min(32, P.no - row0);
        float *dst = P.out + (size_t)w * P.lane_out + (size_t)row0 * P.ldo + col + lane;
        if (col + lane < P.mo)
            for (int q = 0; q < rows; ++q) dst[(size_t)q * P.ldo] = reinterpret_cast<const float *>(box)[32 * q + ((lane + q) & 31)];
        __syncwarp();
    }
}

template <int KIND>
__global__ void __launch_bounds__(DT_THREADS, 1) dots_kernel(const __grid_constant__ CUtensorMap tmx, const __grid_constant__ CUtensorMap tmy,
                                                             const __grid_constant__ CUtensorMap tmo, const __grid_constant__ Dots P)
{
    constexpr bool SCALED = KIND != SKB_BF16;
    // words of scales that a point has in a chunk; an 8-bit cloud's word is that of four chunks
    constexpr int WORDS = KIND == SKB_NV4 ? 4 : KIND == FMT_MX8 ? 1 : 2;
    constexpr uint32_t SF = SCALED ? WORDS * 512 : 0;            // bytes of an operand's scales in a stage
    extern __shared__ __align__(1024) unsigned char smem_dyn[];
    __shared__ __align__(8) unsigned long long bars[3 * DT_STAGES + 5];
    __shared__ __align__(16) float col_points[2][DT_BN];     // read 16 bytes at a time
    __shared__ __align__(16) int col_fars[2][DT_BN / 32];    // whether some of 32 columns' points are not near
    __shared__ uint32_t tmem_holder;
    __shared__ int abort_flag;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    unsigned char *gen = smem_dyn + (base - smem_u32(smem_dyn));
    // operand tiles of all stages, then boxes of results (both want 1024 bytes), then scales
    auto tile_a = [&](int s) { return base + (uint32_t)s * 2 * DT_TILE; };
    const uint32_t boxes = base + DT_STAGES * 2 * DT_TILE, sfs = boxes + 2 * DT_EPI * DT_BOX;
    auto sf_a = [&](int s) { return sfs + (uint32_t)s * 2 * SF; };
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    constexpr int FULL = 0, EMPTY = DT_STAGES, SCALES = 2 * DT_STAGES, ACC = 3 * DT_STAGES, ACC_FREE = ACC + 2, LAST = ACC + 4;
    if (tid == 0) {
        for (int s = 0; s < DT_STAGES; ++s) {
            mbar_init(bar(FULL + s), 1);
            mbar_init(bar(EMPTY + s), 1);
            mbar_init(bar(SCALES + s), 2);
        }
        for (int b = 0; b < 2; ++b) { mbar_init(bar(ACC + b), 1); mbar_init(bar(ACC_FREE + b), DT_EPI); }
        mbar_init(bar(LAST), 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tc_alloc<512>(&tmem_holder);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_holder;

    const int nrt = (P.no + DT_BM - 1) / DT_BM, nct = (P.mo + DT_BN - 1) / DT_BN;
    const long long tiles = (long long)P.W * nrt * nct;
    const int chunks = (P.row_bytes + 127) / 128;
    auto where = [&](long long t, int &w, int &i0, int &j0) {
        const int per_lane = nrt * nct, r = (int)(t % per_lane);
        w = (int)(t / per_lane);
        i0 = r / nct * DT_BM;
        j0 = r % nct * DT_BN;
    };

    if (warp == 0) {
        if (lane == 0) {
            int s = 0, ph = 1;
            unsigned issued = 0;                                  // stages with a load that may still be on its way
            bool ok = true;
            for (long long t = blockIdx.x; ok && t < tiles; t += gridDim.x) {
                int w, i0, j0;
                where(t, w, i0, j0);
                for (int c = 0; c < chunks; ++c) {
                    if (!(ok = mbar_wait(bar(EMPTY + s), ph, &abort_flag))) break;
                    mbar_expect_tx(bar(FULL + s), 2 * DT_TILE);
                    tma_load_points(tile_a(s), &tmx, c * 128, i0, w, bar(FULL + s));
                    tma_load_points(tile_a(s) + DT_TILE, &tmy, c * 128, j0, w, bar(FULL + s));
                    issued = (issued & ~(1u << (s + 16))) | (1u << s) | ((unsigned)(ph ^ 1) << (s + 16));
                    if (++s == DT_STAGES) { s = 0; ph ^= 1; }
                }
            }
            // nothing may land in shared memory after the block has gone: the last load of every stage, with a bound of its own
            int unused = 0;
            for (int q = 0; q < DT_STAGES; ++q)
                if (issued >> q & 1u) mbar_wait(bar(FULL + q), issued >> (q + 16) & 1u, &unused);
        }
    } else if (warp == 1) {
        // (the whole warp walks through the chunks, so that descriptors are uniform; one thread issues: a thread by itself takes longer to form them than the
        // instructions take)
        int s = 0, ph = 0, b = 0, bph = 1;
        bool ok = true;
        for (long long t = blockIdx.x; ok && t < tiles; t += gridDim.x) {
            for (int c = 0; c < chunks; ++c) {
                const bool starts = c % DT_PART<KIND> == 0, ends = (c + 1) % DT_PART<KIND> == 0 || c + 1 == chunks;
                if (starts) {
                    ok = mbar_wait(bar(ACC_FREE + b), bph, &abort_flag);
                    if (!(ok = __all_sync(0xffffffffu, ok))) break;
                }
                ok = mbar_wait(bar(FULL + s), ph, &abort_flag);
                if constexpr (SCALED) ok = ok && mbar_wait(bar(SCALES + s), ph, &abort_flag);
                if (!(ok = __all_sync(0xffffffffu, ok))) break;
                tc_fence_after();
                const uint32_t acc = tmem + b * DT_BN, sf = tmem + DT_SF_COL + s * DT_SF_STRIDE;
                const uint64_t da = tc_desc(tile_a(s)), db = tc_desc(tile_a(s) + DT_TILE);
                const int left = P.row_bytes - c * 128;           // 32 bytes of a point to an instruction
                if (elected()) {
                    if constexpr (SCALED) {
#pragma unroll
                        for (int q = 0; q < WORDS; ++q) {
                            scales_to_tmem(sf + 4 * q, sf_a(s) + 512 * q);
                            scales_to_tmem(sf + 16 + 4 * q, sf_a(s) + SF + 512 * q);
                        }
                    }
                    auto one = [&](int q, uint32_t accumulate) {
                        const int word = KIND == SKB_NV4 ? q : KIND == FMT_MX8 ? 0 : q / 2;
                        // which of a word's four scales: the first or second two, or the chunk's
                        const uint32_t part = KIND == SKB_MX4 ? (uint32_t)(q & 1) * 2u : KIND == FMT_MX8 ? (uint32_t)(c & 3) : 0u;
                        dots_mma<KIND>(acc, da + 2 * q, db + 2 * q, dots_idesc<KIND>() | part << 29 | part << 4, sf + 4 * word, sf + 16 + 4 * word, accumulate);
                    };
                    one(0, !starts);
                    if (left >= 128) {
#pragma unroll
                        for (int q = 1; q < 4; ++q) one(q, 1u);
                    } else {
#pragma unroll
                        for (int q = 1; q < 4; ++q)
                            if (32 * q < left) one(q, 1u);
                    }
                    tc_commit(bar(EMPTY + s));
                    if (ends) tc_commit(bar(ACC + b));
                }
                __syncwarp();
                if (++s == DT_STAGES) { s = 0; ph ^= 1; }
                if (ends) {
                    b ^= 1;
                    if (b == 0) bph ^= 1;
                }
            }
        }
        // what was issued is over before tensor memory is given back
        if (elected()) {
            tc_commit(bar(LAST));
            int unused = 0;
            mbar_wait(bar(LAST), 0, &unused);
        }
        __syncwarp();
    } else if (warp < 6) {
        if constexpr (SCALED) {
            const int op = (warp - 2) & 1, turn = (warp - 2) >> 1;     // operand; every other chunk
            const uint8_t *src = op ? P.sy : P.sx;
            const int npts = op ? P.m : P.n, words = P.sb / 4;
            long long k = 0;                                          // chunks so far
            bool ok = true;
            for (long long t = blockIdx.x; ok && t < tiles; t += gridDim.x) {
                int w, i0, j0;
                where(t, w, i0, j0);
                const int p0 = op ? j0 : i0;
                for (int c = 0; c < chunks; ++c, ++k) {
                    if ((int)(k & 1) != turn) continue;
                    const int c0 = KIND == FMT_MX8 ? c / 4 : c * WORDS;
                    uint32_t v[4][WORDS];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int p = p0 + lane + 32 * q;
                        const uint32_t *row = reinterpret_cast<const uint32_t *>(src + ((size_t)w * npts + min(p, npts - 1)) * P.sb);
#pragma unroll
                        for (int a = 0; a < WORDS; ++a) v[q][a] = p < npts && c0 + a < words ? __ldg(row + c0 + a) : 0u;
                    }
                    const int s = (int)(k % DT_STAGES);
                    ok = mbar_wait(bar(EMPTY + s), (uint32_t)((k / DT_STAGES) & 1) ^ 1u, &abort_flag);
                    if (!(ok = __all_sync(0xffffffffu, ok))) break;
                    // a word of scales of 128 points: row l of 32 holds the words of points l, l + 32, l + 64, l + 96
                    uint4 *dst = reinterpret_cast<uint4 *>(gen + (sf_a(s) - base) + op * SF) + lane;
#pragma unroll
                    for (int a = 0; a < WORDS; ++a) dst[32 * a] = make_uint4(v[0][a], v[1][a], v[2][a], v[3][a]);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(SCALES + s));
                }
            }
        }
    } else {
        // the lanes of tensor memory that this warp may read, and its half of a tile's columns
        const int quarter = warp & 3, half = (warp - 6) >> 2, e = (warp - 6) * 32 + lane;
        const uint32_t box0 = boxes + (uint32_t)(warp - 6) * 2 * DT_BOX;
        unsigned char *gbox0 = gen + (box0 - base);
        int b = 0, ph = 0, turn = 0, even = 0;
        bool ok = true;
        // powers of two of this thread's row, and of a column for all, of the tile that comes next (1: none).  All warps want them at the
        // start of a tile, to know whether it has far ones: loaded there 4 lanes of 4096 x 4096 x 512 take 72 us, a tile ahead 64
        float rp_next = 1.f, cp_next = 1.f;
        auto next_points = [&](long long t) {
            if (t >= tiles) return;
            int w, i0, j0;
            where(t, w, i0, j0);
            const int row = i0 + quarter * 32 + lane, col = j0 + e;
            rp_next = row < P.n ? __ldg(P.px + (size_t)w * P.n + row) : 1.f;
            cp_next = e < DT_BN && col < P.m ? __ldg(P.py + (size_t)w * P.m + col) : 1.f;
        };
        if constexpr (KIND == SKB_NV4) next_points(blockIdx.x);
        for (long long t = blockIdx.x; t < tiles; t += gridDim.x) {
            int w, i0, j0;
            where(t, w, i0, j0);
            float rp = 1.f;
            bool far = false;
            if constexpr (KIND == SKB_NV4) {
                // (the buffer of two tiles ago: its readers have passed the barrier of the last tile)
                const float cp = cp_next;
                rp = rp_next;
                next_points(t + gridDim.x);
                if (e < DT_BN) col_points[even][e] = cp;
                const bool col_far = __any_sync(0xffffffffu, far_point(cp)), row_far = __any_sync(0xffffffffu, far_point(rp));
                if (lane == 0 && warp < 10) col_fars[even][warp - 6] = col_far;
                asm volatile("bar.sync 1, %0;" ::"n"(DT_EPI * 32) : "memory");
                far = row_far || (col_fars[even][0] | col_fars[even][1] | col_fars[even][2] | col_fars[even][3]) != 0;
            }
            const int c_first = half * (DT_BN / 2);
            // (an accumulator that is written again goes back when it has been read)
            auto wait_acc = [&] {
                ok = ok && mbar_wait(bar(ACC + b), ph, &abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                tc_fence_after();
                return tmem + (uint32_t)(quarter << 21) + b * DT_BN + c_first;
            };
            auto free_acc = [&] {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(ACC_FREE + b));
                b ^= 1;
                if (b == 0) ph ^= 1;
            };
            uint32_t held[SCALED ? 1 : 2][32], src = 0;
            if constexpr (SCALED) {
                src = wait_acc();
                if (KIND == SKB_NV4 && far) {
                    far_tile(P, gbox0 + turn * DT_BOX, src, ok, w, i0 + quarter * 32, j0 + c_first, rp, &col_points[even][c_first], lane);
                    free_acc();
                    even ^= 1;
                    continue;
                }
            } else {
                // sums of the parts, added; the 64 columns stay in registers (4-bit kinds, whose products are one part, are faster by
                // boxes: 64 lanes of 1024 x 1024 x 512 56 us so, 75 this way)
                for (int c = 0; c < chunks; c += DT_PART<KIND>) {
                    src = wait_acc();
                    if (!ok) {
#pragma unroll
                        for (int q = 0; q < 64; ++q) held[q / 32][q % 32] = 0x7fffffffu;
                    } else if (c == 0) {
                        tc_ld32_issue(src, held[0]);
                        tc_ld32_issue(src + 32, held[1]);
                        tc_ld_wait(held[0]);
                        tc_ld_wait(held[1]);
                    } else {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t v[32];
                            tc_ld32_issue(src + 32 * h, v);
                            tc_ld_wait(v);
#pragma unroll
                            for (int q = 0; q < 32; ++q) held[h][q] = __float_as_uint(__uint_as_float(held[h][q]) + __uint_as_float(v[q]));
                        }
                    }
                    free_acc();
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c0 = c_first + 32 * h;
                // (a box that is written is stored: the wait below counts stores, and one that were left out would let the next
                // box but one be written while it is read)
                if (j0 + c0 >= P.mo || i0 + quarter * 32 >= P.no) break;
                uint32_t (&r)[32] = held[SCALED ? 0 : h];
                if constexpr (SCALED) {
                    if (ok) {
                        tc_ld32_issue(src + 32 * h, r);
                        tc_ld_wait(r);
                    } else {
#pragma unroll
                        for (int q = 0; q < 32; ++q) r[q] = 0x7fffffffu;
                    }
                }
                if constexpr (KIND == SKB_NV4) {
#pragma unroll
                    for (int q = 0; q < 32; q += 4) {
                        const float4 p = *reinterpret_cast<const float4 *>(&col_points[even][c0 + q]);
                        r[q] = __float_as_uint(__uint_as_float(r[q]) * rp * p.x);
                        r[q + 1] = __float_as_uint(__uint_as_float(r[q + 1]) * rp * p.y);
                        r[q + 2] = __float_as_uint(__uint_as_float(r[q + 2]) * rp * p.z);
                        r[q + 3] = __float_as_uint(__uint_as_float(r[q + 3]) * rp * p.w);
                    }
                }
                // the store before the last one has read its box
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                __syncwarp();
                unsigned char *box = gbox0 + turn * DT_BOX;
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    *reinterpret_cast<uint4 *>(box + lane * 128 + ((q ^ (lane & 7)) << 4)) = make_uint4(r[4 * q], r[4 * q + 1], r[4 * q + 2], r[4 * q + 3]);
                if (P.tma_out) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) tma_store_box(&tmo, box0 + turn * DT_BOX, j0 + c0, i0 + quarter * 32, w);
                } else {
                    __syncwarp();
                    const int rows = min(32, P.no - (i0 + quarter * 32));
                    float *dst = P.out + (size_t)w * P.lane_out + (size_t)(i0 + quarter * 32) * P.ldo + j0 + c0 + lane;
                    if (j0 + c0 + lane < P.mo)
                        for (int q = 0; q < rows; ++q)
                            dst[(size_t)q * P.ldo] = *reinterpret_cast<const float *>(box + q * 128 + (((lane >> 2) ^ (q & 7)) << 4) + (lane & 3) * 4);
                    __syncwarp();
                }
                turn ^= 1;
            }
            if constexpr (SCALED) free_acc();
            even ^= 1;
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tc_dealloc<512>(tmem);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encoder()
{
    static const EncodeTiledFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess ? (EncodeTiledFn)p : (EncodeTiledFn) nullptr;
    }();
    return fn;
}
bool make_map(CUtensorMap *tm, CUtensorMapDataType type, const void *base, cuuint64_t inner, cuuint64_t rows, cuuint64_t W, cuuint64_t pitch,
              cuuint64_t lane_pitch, cuuint32_t box_inner, cuuint32_t box_rows)
{
    const cuuint64_t dims[3] = {inner, rows, W}, strides[2] = {pitch, lane_pitch};
    const cuuint32_t box[3] = {box_inner, box_rows, 1}, step[3] = {1, 1, 1};
    return encoder()(tm, type, 3, const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int KIND>
skb_status launch_kind(const CUtensorMap &tx, const CUtensorMap &ty, const CUtensorMap &to, const Dots &P, int sms, cudaStream_t st)
{
    constexpr int sf = KIND == SKB_BF16 ? 0 : KIND == SKB_NV4 ? 2048 : KIND == FMT_MX8 ? 512 : 1024;
    constexpr int smem = DT_STAGES * (2 * (int)DT_TILE + 2 * sf) + 2 * DT_EPI * (int)DT_BOX + 1024;
    cudaFuncSetAttribute(dots_kernel<KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    const long long tiles = (long long)P.W * ((P.no + DT_BM - 1) / DT_BM) * ((P.mo + DT_BN - 1) / DT_BN);
    dots_kernel<KIND><<<(unsigned)(tiles < sms ? tiles : sms), DT_THREADS, smem, st>>>(tx, ty, to, P);
    return op_launched("products");
}

}  // namespace

bool points_map(CUtensorMap *tm, const void *codes, int row_bytes, int npts, int W, int box_points)
{
    const size_t rb = row_bytes;
    return encoder() && make_map(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, rb, npts, W, rb, rb * npts, 128, box_points);
}

bool staged_map(CUtensorMap *tm, const void *base, size_t rows)
{
    const cuuint64_t dims[2] = {64, rows}, strides[1] = {128};
    const cuuint32_t box[2] = {64, 64}, step[2] = {1, 1};
    return encoder() && encoder()(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                  CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool queries_map(CUtensorMap *tm, const void *x, int d, int n, int W)
{
    const size_t rb = 2 * (size_t)d;
    return encoder() && make_map(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, x, d, n, W, rb, rb * n, 64, 128);
}

DotsCloud dots_cloud(const void *base, const Cloud4 &c, int dtype, int d, size_t row)
{
    if (dtype == SKB_BF16) return {(const uint16_t *)base + row * d, nullptr, nullptr, 2 * d, 0};
    return {c.codes + row * c.cb, c.scales + row * c.sb, c.points ? c.points + row : nullptr, c.cb, c.sb};
}

skb_status launch_dots(const DotsCloud &x, const DotsCloud &y, int dtype, int W, int n, int m, float *out, long long ldo, cudaStream_t st,
                       int n_out, int m_out)
{
    if (!encoder()) return op_fail(SKB_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
    int dev = 0, sms = 0;
    cudaGetDevice(&dev);
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return op_launched("device");
    Dots P = {};
    P.W = W; P.n = n; P.m = m;
    P.no = n_out > n ? n_out : n; P.mo = m_out > m ? m_out : m;
    P.out = out; P.ldo = ldo; P.lane_out = ldo * P.no;
    P.sx = x.scales; P.sy = y.scales; P.px = x.points; P.py = y.points;
    P.row_bytes = x.row_bytes; P.sb = x.sb;
    const void *cx = x.data, *cy = y.data;
    P.tma_out = ldo % 4 == 0 && (uintptr_t)out % 16 == 0;
    CUtensorMap tx, ty, to = {};
    const size_t rb = P.row_bytes;
    if (!make_map(&tx, CU_TENSOR_MAP_DATA_TYPE_UINT8, cx, rb, n, W, rb, rb * n, 128, DT_BM) ||
        !make_map(&ty, CU_TENSOR_MAP_DATA_TYPE_UINT8, cy, rb, m, W, rb, rb * m, 128, DT_BN) ||
        (P.tma_out && !make_map(&to, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, out, P.mo, P.no, W, ldo * 4, ldo * 4 * P.no, 32, 32)))
        return op_fail(SKB_ERR_CUDA, "cuTensorMapEncodeTiled failed");
    if (dtype == SKB_BF16) return launch_kind<SKB_BF16>(tx, ty, to, P, sms, st);
    if (dtype == SKB_MX4) return launch_kind<SKB_MX4>(tx, ty, to, P, sms, st);
    if (dtype == FMT_MX8) return launch_kind<FMT_MX8>(tx, ty, to, P, sms, st);
    return launch_kind<SKB_NV4>(tx, ty, to, P, sms, st);
}

}  // namespace skb

using namespace skb;

extern "C" skb_status sinkhorn_cloud4_dots(const void *x, const void *y, int W, int n, int m, int d, int format, float *out, void *stream)
{
    if (!x || !y || !out) return op_fail(SKB_ERR_NULL, "x, y and out are required");
    if (const char *why = cloud4_refused(W, n, d, format)) return op_fail(SKB_ERR_SHAPE, why);
    if (const char *why = cloud4_refused(W, m, d, format)) return op_fail(SKB_ERR_SHAPE, why);
    if ((uintptr_t)x % 256 || (uintptr_t)y % 256) return op_fail(SKB_ERR_WORKSPACE, "x and y must be 256-byte aligned");
    if ((uintptr_t)out % 4) return op_fail(SKB_ERR_WORKSPACE, "out must be 4-byte aligned");
    const Cloud4 a = cloud4_view(x, (size_t)W * n, d, format), b = cloud4_view(y, (size_t)W * m, d, format);
    return launch_dots(dots_cloud(x, a, format, d, 0), dots_cloud(y, b, format, d, 0), format, W, n, m, out, m, (cudaStream_t)stream);
}
