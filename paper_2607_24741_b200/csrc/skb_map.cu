// Images of query points under the entropic map of a target cloud held in 8 bits: attention over a stored bank,
//      out_i = sum_j w_ij v_j,   w_i = softmax over j of (g_j - |x_i - y_j|^2) / eps,
// in one pass over the bank: exponents as k (2 x.y + g_j - |y_j|^2), k = log2(e) / eps, against a running maximum (|x_i|^2 is the same for all j).
//
// map_rows_kernel, here: few queries, the serving form.  Eight or sixteen queries and a part of a lane's bank to a block of four warps, two
// to three blocks an SM.  Bounded by memory: every code is read once (by one block of queries), n <= 16 makes at most 64 flop of a byte.
//   load     64 points at a time, 128 dimensions of them a slot of 8 KB, by TMA (128-byte swizzle, points past the end are zeros) into a ring
//            of slots that holds two to eight tiles
//   scores   a warp takes 16 points: codes to f16 in registers (exact), mma.sync with the queries' f16 (a power of two for each query: its
//            largest value is 2^14, so nothing of bf16's eight bits is lost above 2^-38 of it), 128 dimensions at a time, whose sums are multiplied
//            by the block's power of two in fp32
//   softmax  all threads: exponentials in fp32 against the running maximum of the query, sums in fp32
//   images   weights times the values' powers of two, less the tile's largest, in f16 (11 bits; what is below 2^-25 of the largest value of
//            a tile's 64 points is lost), a warp takes 32 dimensions of every 128: bytes of two points side by side by prmt, to f16, mma.sync; sums of a
//            tile are added in fp32
// Several blocks that share a lane's bank leave (maximum, sum, image), which map_join_kernel adds up in the order of the parts.
// The matrix instructions are mma.sync, whose operands come from registers: eight queries are an eighth of a tcgen05 tile, and codes
// would have to go back to shared memory as f16 first.
#include <cuda.h>
#include <cuda_runtime.h>
#include <string>

#include "skb_cloud_io.cuh"
#include "skb_map.cuh"
#include "skb_operators.h"
#include "skb_tmem.cuh"

namespace skb {
namespace {

constexpr int MR_THREADS = 128, MR_T = 64;                    // points of a tile
constexpr uint32_t MR_SLOT = MR_T * 128;
constexpr int MR_MAX_SLOTS = 20, MR_PSTRIDE = 72;             // f16 from query to query: rows end up four banks apart

__device__ __forceinline__ float ex2f(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// codes of the low or high half of a word as f16
__device__ __forceinline__ uint32_t half_lo(uint32_t w)
{
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t half_hi(uint32_t w)
{
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint16_t f16_bits(float v)
{
    uint16_t r;
    asm("cvt.rn.f16.f32 %0, %1;" : "=h"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void tma_points(uint32_t dst, const CUtensorMap *tm, int byte, int point, int lane, uint32_t mbar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(byte), "r"(point), "r"(lane), "r"(mbar) : "memory");
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// blocks that an SM is to hold: their waits, for barriers as for memory, are each other's time
template <int NG, int UNITS> constexpr int MR_BLOCKS = NG * UNITS <= 4 ? 4 : NG * UNITS <= 8 ? 3 : 2;

// NG groups of eight queries; UNITS blocks of 128 dimensions of values
template <int NG, int UNITS>
__global__ void __launch_bounds__(MR_THREADS, MR_BLOCKS<NG, UNITS>) map_rows_kernel(const __grid_constant__ CUtensorMap tmy, const __grid_constant__ CUtensorMap tmv,
                                                              const __grid_constant__ Map P, const int slots)
{
    constexpr int Q = 8 * NG;
    extern __shared__ __align__(1024) unsigned char smem_dyn[];
    __shared__ __align__(8) unsigned long long bars[MR_MAX_SLOTS];
    __shared__ __align__(16) float s_arg[Q][MR_T];
    __shared__ __align__(16) uint16_t s_p[UNITS][Q][MR_PSTRIDE];
    __shared__ float s_max[4][Q], s_run[Q], s_fac[Q], s_kx[Q], s_sum[MR_THREADS / 32][Q];
    __shared__ __align__(8) uint8_t s_scale[MR_T][8];
    __shared__ int s_top[4][UNITS];
    __shared__ double s_xx[Q];
    __shared__ int abort_flag;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = lane >> 2, c = lane & 3;
    const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    unsigned char *gen = smem_dyn + (base - smem_u32(smem_dyn));
    const int split = blockIdx.x, q0 = blockIdx.y * Q, w = blockIdx.z;
    const int nby = (P.d + 127) / 128, nbv = P.own_values ? (P.dv + 127) / 128 : 0, per_tile = nby + nbv;
    uint2 *xf = reinterpret_cast<uint2 *>(gen + (size_t)slots * MR_SLOT);      // [NG][8 nby][32] fragments of the queries
    auto bar = [&](int s) { return smem_u32(&bars[s]); };

    const int len = map_length(P, w), tiles = (len + MR_T - 1) / MR_T;
    const int t0 = (int)((long long)tiles * split / P.splits), t1 = (int)((long long)tiles * (split + 1) / P.splits);
    if (tid == 0) {
        for (int s = 0; s < slots; ++s) mbar_init(bar(s), 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    // slots are filled in the order of tiles and their blocks: the bank's, then those of values of their own.  (Slots, tiles and phases are counted
    // on: divisions would be half of the instructions.)
    int in_tile = t0, in_block = 0, in_slot = 0;                              // (thread 0) what comes into a slot next
    auto issue = [&](int count) {
        for (; count > 0 && in_tile < t1; --count) {
            mbar_expect_tx(bar(in_slot), MR_SLOT);
            if (in_block < nby) tma_points(base + in_slot * MR_SLOT, &tmy, in_block * 128, in_tile * MR_T, w, bar(in_slot));
            else tma_points(base + in_slot * MR_SLOT, &tmv, (in_block - nby) * 128, in_tile * MR_T, w, bar(in_slot));
            if (++in_block == per_tile) { in_block = 0; ++in_tile; }
            if (++in_slot == slots) in_slot = 0;
        }
    };
    if (tid == 0) issue(slots);

    // the queries: a power of two, the squared length, then f16 in the order of the matrix instruction's fragments.  A warp takes every fourth.
    const double k = map_scale(P, w);
    for (int q = warp; q < Q; q += 4) {
        const bool live = q0 + q < P.n;
        const uint16_t *x = P.x + ((size_t)w * P.n + (live ? q0 + q : 0)) * P.d;
        float top = 0.f;
        bool bad = false;
        double xx = 0.0;
        if (live)
            for (int i = lane; i < P.d; i += 32) {
                const float v = __uint_as_float((uint32_t)x[i] << 16);
                bad |= !(fabsf(v) <= 3.402823466e38f);
                top = fmaxf(top, fabsf(v));
                xx += (double)v * (double)v;
            }
#pragma unroll
        for (int off = 16; off; off /= 2) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            xx += __shfl_xor_sync(0xffffffffu, xx, off);
        }
        bad = __any_sync(0xffffffffu, bad);
        const int ex = top > 0.f && !bad ? max(exponent_of(top) - 14, -126) : 0;
        const float inv = power_of_two(-ex);
        // fragment of eight dimensions 64 b + 16 c + 4 s .. + 3: lane (query, c) of step 4 b + s
        for (int i = lane; i < 32 * nby; i += 32) {                            // words of four dimensions
            uint32_t h[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int dim = 4 * i + e;
                uint32_t bits = 0;
                if (live && dim < P.d) bits = bad ? 0x7fffu : f16_bits(__uint_as_float((uint32_t)x[dim] << 16) * inv);
                h[e / 2] |= bits << (16 * (e & 1));
            }
            const int b = i / 16, cc = i / 4 % 4, s = i % 4;
            xf[((q >> 3) * 8 * nby + 4 * b + s) * 32 + 4 * (q & 7) + cc] = make_uint2(h[0], h[1]);
        }
        if (lane == 0) {
            s_kx[q] = (float)(2.0 * k * (double)power_of_two(ex));
            s_xx[q] = xx;
            s_run[q] = -INFINITY;
        }
    }

    float out[UNITS][NG][2][4];
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
        for (int a = 0; a < NG; ++a)
#pragma unroll
            for (int i = 0; i < 8; ++i) out[u][a][i / 4][i & 3] = 0.f;
    float sum[Q / 2];                                                          // of this thread's point of a tile, for every other query
#pragma unroll
    for (int i = 0; i < Q / 2; ++i) sum[i] = 0.f;

    // this lane's two points of a tile (rows of the fragment are points in an order that keeps shared memory's banks apart)
    const int pa = 16 * warp + ((row >> 1) | ((row & 1) << 2)), pb = pa + 8;
    const uint2 none = make_uint2(0u, 0u);
    struct Point {
        float term;
        uint2 sy, sv;
    };
    auto fetch = [&](int t, int p) {
        Point r = {-INFINITY, none, none};
        const int j = t * MR_T + p;
        if (j >= len) return r;
        const size_t at = (size_t)w * P.m + j;
        r.term = map_term(k, P.g ? P.g[at] : 0.0, P.y.norms[at]);
        const uint32_t *sy = reinterpret_cast<const uint32_t *>(P.y.scales + at * P.y.sb);
        r.sy = make_uint2(sy[0], P.y.sb > 4 ? sy[1] : 0u);
        if (P.own_values) {
            const uint32_t *sv = reinterpret_cast<const uint32_t *>(P.v.scales + at * P.v.sb);
            r.sv = make_uint2(sv[0], P.v.sb > 4 ? sv[1] : 0u);
        } else r.sv = r.sy;
        return r;
    };
    auto byte_of = [](uint2 s, int b) { return ((b < 4 ? s.x : s.y) >> (8 * (b & 3))) & 255u; };
    Point na, nb;
    if (t0 < t1) { na = fetch(t0, pa); nb = fetch(t0, pb); }
    __syncthreads();

    int slot0 = 0;                                                            // of a tile's first block, and the phase it is filled in
    uint32_t phase = 0;
    bool ok = true;
    for (int t = t0; t < t1; ++t) {
        const Point A = na, Bp = nb;
        if (t + 1 < t1) { na = fetch(t + 1, pa); nb = fetch(t + 1, pb); }
        auto slot_of = [&](int b) { return slot0 + b < slots ? slot0 + b : slot0 + b - slots; };
        auto wait = [&](int b) {
            const int i = slot_of(b);
            ok = mbar_wait(bar(i), phase ^ (slot0 + b < slots ? 0u : 1u), &abort_flag) && ok;
            return gen + i * MR_SLOT;
        };
        // ---- scores
        float s[NG][4];
#pragma unroll
        for (int a = 0; a < NG; ++a)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[a][i] = 0.f;
        for (int b = 0; b < nby; ++b) {
            const unsigned char *slot = wait(b);
            float acc[NG][4];
#pragma unroll
            for (int a = 0; a < NG; ++a)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[a][i] = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 ra = *reinterpret_cast<const uint4 *>(slot + pa * 128 + (((4 * h + c) ^ (pa & 7)) << 4));
                const uint4 rb = *reinterpret_cast<const uint4 *>(slot + pb * 128 + (((4 * h + c) ^ (pb & 7)) << 4));
                const uint32_t wa[4] = {ra.x, ra.y, ra.z, ra.w}, wb[4] = {rb.x, rb.y, rb.z, rb.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t a0 = half_lo(wa[q]), a1 = half_lo(wb[q]), a2 = half_hi(wa[q]), a3 = half_hi(wb[q]);
#pragma unroll
                    for (int a = 0; a < NG; ++a) {
                        const uint2 x = xf[(a * 8 * nby + 8 * b + 4 * h + q) * 32 + lane];
                        mma16816(acc[a], a0, a1, a2, a3, x.x, x.y);
                    }
                }
            }
            const float fa = e8m0_value(byte_of(A.sy, b)), fb = e8m0_value(byte_of(Bp.sy, b));
#pragma unroll
            for (int a = 0; a < NG; ++a) {
                s[a][0] = fmaf(acc[a][0], fa, s[a][0]);
                s[a][1] = fmaf(acc[a][1], fa, s[a][1]);
                s[a][2] = fmaf(acc[a][2], fb, s[a][2]);
                s[a][3] = fmaf(acc[a][3], fb, s[a][3]);
            }
        }
#pragma unroll
        for (int a = 0; a < NG; ++a)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int q = 8 * a + 2 * c + i;
                const float kx = s_kx[q];
                // (what a masked point's codes hold does not matter)
                const float va = A.term == -INFINITY ? -INFINITY : fmaf(s[a][i], kx, A.term), vb = Bp.term == -INFINITY ? -INFINITY : fmaf(s[a][2 + i], kx, Bp.term);
                s_arg[q][pa] = va;
                s_arg[q][pb] = vb;
                float top = fmaxf(va, vb);
#pragma unroll
                for (int off = 4; off < 32; off *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
                if (row == 0) s_max[warp][q] = top;
            }
        // the values' scales, and the largest exponent of the tile in each block (of points that are masked or NaN: none)
        if (c == 0) {
            *reinterpret_cast<uint2 *>(s_scale[pa]) = A.sv;
            *reinterpret_cast<uint2 *>(s_scale[pb]) = Bp.sv;
        }
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const uint32_t ea = byte_of(A.sv, u), eb = byte_of(Bp.sv, u);
            const uint32_t one = max(A.term == -INFINITY || ea == 255u ? 0u : ea, Bp.term == -INFINITY || eb == 255u ? 0u : eb);
            const uint32_t top = __reduce_max_sync(0xffffffffu, one);
            if (lane == 0) s_top[warp][u] = (int)top;
        }
        __syncthreads();
        // ---- softmax: thread = point and every other query
        {
            const int p = tid & 63, other = tid >> 6;
            uint32_t scale[UNITS];
            const uint2 sv = *reinterpret_cast<const uint2 *>(s_scale[p]);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int e = (int)byte_of(sv, u), top = max(max(s_top[0][u], s_top[1][u]), max(s_top[2][u], s_top[3][u]));
                // a power of two (0: below fp32's), or NaN; masked points have weights of zero
                scale[u] = e == 255 ? 0x7fffffffu : e > top ? 0u : e - top + 127 <= 0 ? 0u : (uint32_t)(e - top + 127) << 23;
            }
#pragma unroll
            for (int i = 0; i < Q / 2; ++i) {
                const int q = 2 * i + other;
                const float run = s_run[q], top = fmaxf(fmaxf(fmaxf(s_max[0][q], s_max[1][q]), fmaxf(s_max[2][q], s_max[3][q])), run);
                const float ref = top == -INFINITY ? 0.f : top, arg = s_arg[q][p], fac = ex2f(run - ref);
                const float e = ex2f(arg - ref);
                sum[i] = fmaf(sum[i], fac, e);
                if (p == 0) s_fac[q] = fac;
                const bool masked = arg == -INFINITY;
#pragma unroll
                for (int u = 0; u < UNITS; ++u) s_p[u][q][p] = masked ? (uint16_t)0 : f16_bits(e * __uint_as_float(scale[u]));
            }
        }
        __syncthreads();
        if (tid < Q) {
            const float top = fmaxf(fmaxf(s_max[0][tid], s_max[1][tid]), fmaxf(s_max[2][tid], s_max[3][tid]));
            s_run[tid] = fmaxf(s_run[tid], top);
        }
        // ---- images
        float fac[NG][2];
#pragma unroll
        for (int a = 0; a < NG; ++a) { fac[a][0] = s_fac[8 * a + 2 * c]; fac[a][1] = s_fac[8 * a + 2 * c + 1]; }
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if (128 * u + 32 * warp >= P.dv) break;
            const unsigned char *slot = nbv ? wait(nby + u) : gen + slot_of(u) * MR_SLOT;
            float acc[NG][2][4];
#pragma unroll
            for (int a = 0; a < NG; ++a)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[a][i / 4][i & 3] = 0.f;
#pragma unroll
            for (int kk = 0; kk < MR_T / 16; ++kk) {
                auto word = [&](int p) { return *reinterpret_cast<const uint32_t *>(slot + p * 128 + (((2 * warp + (row >> 2)) ^ (p & 7)) << 4) + (row & 3) * 4); };
                const int p = 16 * kk + 2 * c;
                const uint32_t w0 = word(p), w1 = word(p + 1), w2 = word(p + 8), w3 = word(p + 9);
                const uint32_t l01 = __byte_perm(w0, w1, 0x5140), h01 = __byte_perm(w0, w1, 0x7362);
                const uint32_t l23 = __byte_perm(w2, w3, 0x5140), h23 = __byte_perm(w2, w3, 0x7362);
                const uint32_t a00 = half_lo(l01), a01 = half_hi(l01), a02 = half_lo(l23), a03 = half_hi(l23);
                const uint32_t a10 = half_lo(h01), a11 = half_hi(h01), a12 = half_lo(h23), a13 = half_hi(h23);
#pragma unroll
                for (int a = 0; a < NG; ++a) {
                    const uint16_t *pq = s_p[u][8 * a + row] + p;
                    const uint32_t b0 = *reinterpret_cast<const uint32_t *>(pq), b1 = *reinterpret_cast<const uint32_t *>(pq + 8);
                    mma16816(acc[a][0], a00, a01, a02, a03, b0, b1);
                    mma16816(acc[a][1], a10, a11, a12, a13, b0, b1);
                }
            }
            const int top = max(max(s_top[0][u], s_top[1][u]), max(s_top[2][u], s_top[3][u]));
            const float unit = e8m0_value((uint32_t)top);
#pragma unroll
            for (int a = 0; a < NG; ++a)
#pragma unroll
                for (int i = 0; i < 8; ++i) out[u][a][i / 4][i & 3] = fmaf(out[u][a][i / 4][i & 3], fac[a][i & 1], acc[a][i / 4][i & 3] * unit);
        }
        ok = __syncthreads_and(ok);
        if (!ok) break;
        if (tid == 0) issue(per_tile);
        slot0 += per_tile;
        if (slot0 >= slots) { slot0 -= slots; phase ^= 1u; }
    }
    // nothing may land in shared memory after the block has gone: where a wait ran out, every load that may still be on its way
    if (!ok && tid == 0) {
        int unused = 0, s = slot0;
        uint32_t ph = phase;
        for (int i = 0; i < slots && (s != in_slot || i == 0); ++i) {
            mbar_wait(bar(s), ph, &unused);
            if (++s == slots) { s = 0; ph ^= 1u; }
        }
    }
    // ---- the sums, over points
#pragma unroll
    for (int i = 0; i < Q / 2; ++i) {
#pragma unroll
        for (int off = 16; off; off /= 2) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], off);
        if (lane == 0) s_sum[warp][2 * i + (warp >> 1)] = sum[i];
    }
    __syncthreads();
    const float nan = __uint_as_float(0x7fffffffu);
    auto sum_of = [&](int q) { return !ok ? nan : (q & 1) ? s_sum[2][q] + s_sum[3][q] : s_sum[0][q] + s_sum[1][q]; };
    if (tid < Q && q0 + tid < P.n) {
        const size_t r = (size_t)w * P.n + q0 + tid;
        if (P.splits > 1) {
            reinterpret_cast<float2 *>(P.part_ml)[r * P.splits + split] = make_float2(s_run[tid], sum_of(tid));
        } else if (P.lse) P.lse[r] = map_lse(s_run[tid], sum_of(tid), k, s_xx[tid]);
    }
#pragma unroll
    for (int a = 0; a < NG; ++a)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int q = 8 * a + 2 * c + i;
            if (q0 + q >= P.n) continue;
            const size_t r = (size_t)w * P.n + q0 + q;
            const float total_q = sum_of(q), inv = total_q == 0.f ? 0.f : 1.f / total_q;
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int dim = 128 * u + 32 * warp + 4 * row;
                if (dim >= P.dv) continue;
                const float o[4] = {out[u][a][0][i], out[u][a][0][2 + i], out[u][a][1][i], out[u][a][1][2 + i]};
                if (P.splits > 1) {
                    float *dst = P.part_out + (r * P.splits + split) * P.dv + dim;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (dim + e < P.dv) dst[e] = o[e];
                } else {
                    uint16_t *dst = P.out + r * P.dv + dim;
                    const uint32_t lo = bf16_pair(o[0] * inv, o[1] * inv), hi = bf16_pair(o[2] * inv, o[3] * inv);
                    if (P.dv % 4 == 0 && (uintptr_t)P.out % 8 == 0) *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (dim + e < P.dv) dst[e] = (uint16_t)((e < 2 ? lo : hi) >> (16 * (e & 1)));
                }
            }
        }
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
        const float f = ex2f(one.x - ref);
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

template <int NG, int UNITS>
skb_status launch_rows(const CUtensorMap &ty, const CUtensorMap &tv, const Map &P, cudaStream_t st)
{
    const int nby = (P.d + 127) / 128, per_tile = nby + (P.own_values ? (P.dv + 127) / 128 : 0);
    // as many slots as leave room for the blocks that registers allow, a tile at least
    cudaFuncAttributes fa;
    if (cudaFuncGetAttributes(&fa, map_rows_kernel<NG, UNITS>) != cudaSuccess) return op_launched("map");
    const int rest = NG * 8 * nby * 256 + 1024, room = MAP_SM_SMEM / MR_BLOCKS<NG, UNITS> - 1024 - (int)fa.sharedSizeBytes - rest;
    const int slots = min(MR_MAX_SLOTS, max(per_tile, room / (int)MR_SLOT));
    const int smem = slots * (int)MR_SLOT + rest;
    cudaFuncSetAttribute(map_rows_kernel<NG, UNITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    map_rows_kernel<NG, UNITS><<<dim3(P.splits, (P.n + 8 * NG - 1) / (8 * NG), P.W), MR_THREADS, smem, st>>>(ty, tv, P, slots);
    return op_launched("map");
}
template <int NG>
skb_status launch_rows_by_depth(const CUtensorMap &ty, const CUtensorMap &tv, const Map &P, cudaStream_t st)
{
    if (P.dv <= 128) return launch_rows<NG, 1>(ty, tv, P, st);
    if (P.dv <= 256) return launch_rows<NG, 2>(ty, tv, P, st);
    if (P.dv <= 512) return launch_rows<NG, 4>(ty, tv, P, st);
    return launch_rows<NG, 8>(ty, tv, P, st);
}

// queries up to which the matrix unit's tiles of 128 are too empty
constexpr int MAP_ROWS_MAX = 32;

const char *map_refused(int W, int n, int m, int d, int dv)
{
    if (W < 1 || n < 1 || m < 1 || d < 1) return "W, n, m and d must be >= 1";
    if (W > 65535 || n > 262143 || m > 262143) return "W at most 65535, n and m at most 262143";
    if (d > CLOUD8_MAX_D || dv > CLOUD8_MAX_D || dv < 0) return "d and dv must be at most 1024";
    return nullptr;
}
// Which kernel, and into how many parts a lane's bank goes: enough to fill the device, of a few tiles at least.
struct MapPlan {
    bool tiles;
    int splits;
};
int rows_blocks(int n, int dv)
{
    const int units = dv <= 128 ? 1 : dv <= 256 ? 2 : dv <= 512 ? 4 : 8, work = (n <= 8 ? 1 : 2) * units;
    return work <= 4 ? 4 : work <= 8 ? 3 : 2;                     // MR_BLOCKS
}
MapPlan map_plan(int W, int n, int m, int d, int dv, int sms)
{
    MapPlan p;
    p.tiles = n > MAP_ROWS_MAX && d <= MAP_TILES_MAX_D;
    const long long blocks = p.tiles ? (long long)W * (n > 128 ? (n + 255) / 256 * 2 : 1) * ((dv + 255) / 256) : (long long)W * (n <= 8 ? 1 : (n + 15) / 16);
    const long long tiles = p.tiles ? (m + 127) / 128 : (m + MR_T - 1) / MR_T;
    long long s = p.tiles ? sms / blocks : (long long)rows_blocks(n, dv) * sms / blocks;
    if (s > tiles / 2) s = tiles / 2;
    p.splits = (int)(s < 1 ? 1 : s > 128 ? 128 : s);
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
    const MapPlan p = map_plan(W, n, m, d, dv, MAP_MAX_SMS);
    return 256 + map_parts_bytes(W, n, dv, p.splits) + (p.tiles ? pad256(map_staged_bytes(W, m, d, dv, own_values)) : 0);
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
    int dev = 0, sms = 0;
    cudaGetDevice(&dev);
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return op_launched("device");
    Map P = {};
    P.x = (const uint16_t *)x;
    P.y = cloud8_view(y, (size_t)W * m, d);
    P.v = v ? cloud8_view(v, (size_t)W * m, dv) : P.y;
    P.g = g; P.eps = eps; P.lengths = lengths; P.out = (uint16_t *)out; P.lse = lse;
    P.W = W; P.n = n; P.m = m; P.d = d; P.dv = depth; P.own_values = v != nullptr;
    const MapPlan plan = map_plan(W, n, m, d, depth, sms < MAP_MAX_SMS ? sms : MAP_MAX_SMS);
    P.splits = plan.splits;
    P.part_ml = (float *)workspace;
    P.part_out = (float *)((char *)workspace + pad256((size_t)W * n * P.splits * 8));
    void *room = (char *)workspace + map_parts_bytes(W, n, depth, P.splits);
    CUtensorMap ty, tv;
    if (!plan.tiles && (!points_map(&ty, P.y.codes, P.y.cb, m, W, MR_T) || !points_map(&tv, P.v.codes, P.v.cb, m, W, MR_T)))
        return op_fail(SKB_ERR_CUDA, "cuTensorMapEncodeTiled failed");
    const skb_status rc = plan.tiles ? launch_map_tiles(P, room, sms, (cudaStream_t)stream) : n <= 8 ? launch_rows_by_depth<1>(ty, tv, P, (cudaStream_t)stream) : launch_rows_by_depth<2>(ty, tv, P, (cudaStream_t)stream);
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
