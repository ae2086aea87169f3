// Images under the entropic map of a stored cloud for many queries (see skb_map.cu for the mathematics): both products on tcgen05.
//
// map_stage_kernel writes the bank once as bf16 into the workspace, in the order in which the matrix unit wants it in shared memory (blocks of 128 targets by
// 128 dimensions, 32 KB, 128-byte swizzle; the same layout is K-major for the scores and MN-major for the images, so values are not
// transposed), masked targets and what is past the ends as zeros, and the targets' terms.  A value is four bits times a power of two, which
// bf16 holds over all of the clouds' range, so products are those of the values, exactly; f16 would round weights to 11 bits instead of 8, but
// cannot hold values of a bank whose scales differ.  Codes made into bf16 by warps of every block of queries cost more than all else: 64 lanes
// of 1024 x 1024 x 512 took 858 us that way.
//
// map_tiles_kernel: a block takes 128 queries, a part of the bank, and up to 256 dimensions of the values (deeper ones: further blocks, which form the
// scores again).  Per tile of 128 targets
//      S = X . Y^T       bf16, fp32 in tensor memory, two buffers (cut off at every instruction: 2^-20.6 of the magnitudes for every 16 dimensions)
//      P = exp2(2k S + term - reference) in bf16, into S's place in tensor memory
//      O += P . V        bf16, fp32 in tensor memory
// so that the scores of the next tile are formed while this one's exponentials are.  Outputs are bf16; the weights are summed in fp32 before they
// are rounded.
//   warps 0-7    softmax: a thread to a query and half of a tile's targets; the two halves of a query exchange their maxima.  The reference is a
//                whole number, raised only when a tile's maximum passes it by more than 8 (weights up to 2^8 are as good in bf16 as those
//                below 1): O is then multiplied by a power of two, exactly
//   warp 8       loads: bulk copies of 32 KB and of a tile's terms
//   warp 9       matrix instructions, one thread: S of tile t + 1 before O of tile t
// 64 lanes of 1024 queries to 1024 x 512 take 205 us, 22 of them the staging: 206 GFLOP of products (two thirds of them the scores, formed
// for 256 dimensions of the images each) at 1.1 PFLOP/s.  What bounds it: at 128 dimensions the exponentials (128 x 128 of a tile at 16 a clock take as long as
// its products); deeper no unit by itself (the tensor pipe is active for 43 % of 16 lanes' 59 us): a block's queries arrive and its images leave
// with nothing beside them, one block an SM, every eight tiles.
// Weights in bf16 are the choice of one pass of the matrix unit over the values: eight bits as of the images themselves.  Where values average out that
// is felt: images of values of their own with mixed signs are off by 2.4e-3 of their size (rms) where weights in fp32 leave bf16's 1.7e-3.
// Every wait is bounded (skb_tmem.cuh): one that runs out ends all roles, and the block's images are NaN.
#include <cuda.h>
#include <cuda_runtime.h>
#include <string>
#include <type_traits>

#include "skb_f32x2.cuh"
#include "skb_map.cuh"
#include "skb_operators.h"
#include "skb_tmem.cuh"

namespace skb {
namespace {

constexpr int MT_SOFT = 8, MT_LOAD = MT_SOFT, MT_MMA = MT_SOFT + 1, MT_THREADS = (MT_SOFT + 2) * 32;
constexpr uint32_t MT_CHUNK = 128 * 128, MT_BLOCK = 2 * MT_CHUNK;         // 128 points by 64, 128 dimensions of bf16
constexpr int MT_MAX_STAGES = 8;
constexpr uint32_t MT_MISC = 3 * 1024;
constexpr float MT_SLACK = 8.f;
// Tiles whose images are added up in tensor memory.  The matrix unit cuts each of an instruction's 16 products and the sum so far at 2^-25 of the largest,
// and the result at 24 bits: 17 2^-25 + 2^-23 < 2^-20.6 of the sum for every 16 targets, always towards zero.  Over a bank of 262143 that is a
// quarter of a percent of images whose values have one sign; over 64 tiles at most 2^-11.6.
constexpr int MT_CHAIN = 64;

// D fp32, A and B bf16, 128 queries (a pair of blocks: 256) by 128
template <bool PAIR> constexpr uint32_t MT_IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | (((PAIR ? 256u : 128u) >> 4) << 24);
template <bool PAIR> constexpr uint32_t MT_IDESC_V = MT_IDESC<PAIR> | (1u << 16);     // B with its columns next to each other

template <bool PAIR> __device__ __forceinline__ void mma_smem(uint32_t d, uint64_t a, uint64_t b, uint32_t accumulate)
{
    if constexpr (!PAIR) tc_mma(d, a, b, MT_IDESC<PAIR>, accumulate);
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(MT_IDESC<PAIR>), "r"(accumulate) : "memory");
}
// ... with A in tensor memory
template <bool PAIR> __device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t accumulate)
{
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "l"(b), "r"(MT_IDESC_V<PAIR>), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "l"(b), "r"(MT_IDESC_V<PAIR>), "r"(accumulate) : "memory");
}
__device__ __forceinline__ uint32_t in_block(uint32_t a, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync_all()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// an arrival once the matrix instructions so far are done; a pair's, at the barriers of the blocks in the mask
template <bool PAIR> __device__ __forceinline__ void commit(uint32_t mbar, uint16_t mask = 3)
{
    if constexpr (!PAIR) tc_commit(mbar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(mbar), "h"(mask) : "memory");
}
// 64 rows of 128 bytes; the barrier may be the other block's of a pair
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap *tm, int row, uint32_t mbar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(0), "r"(row), "r"(mbar) : "memory");
}
// 128 queries by 64 dimensions
template <bool PAIR> __device__ __forceinline__ void load_queries(uint32_t dst, const CUtensorMap *tm, int dim, int query, int lane, uint32_t mbar)
{
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(dim), "r"(query), "r"(lane), "r"(mbar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(dim), "r"(query), "r"(lane), "r"(mbar) : "memory");
}
// rows of 64 columns (128 bytes), 8-row groups 1024 bytes apart, the next 64 columns a chunk further
__device__ __forceinline__ uint64_t desc_columns(uint32_t saddr)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(MT_CHUNK >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Two codes, in the upper bytes of the halves of p, as bf16 of 2^-120 times their values: their four bits of exponent and three of mantissa are the
// lowest of bf16's eight and the highest of its seven, subnormals among them.
__device__ __forceinline__ uint32_t codes_bf16(uint32_t p) { return ((p >> 4) & 0x07f007f0u) | (p & 0x80008000u); }

// whether all COUNT threads of a barrier say so
template <int COUNT> __device__ __forceinline__ bool all_of(bool ok, int barrier)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbarrier.cta.red.and.pred q, %1, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(barrier), "r"((uint32_t)ok), "n"(COUNT) : "memory");
    return r != 0;
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t mbar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(mbar) : "memory");
}

// The bank as bf16.  A thread takes 16 codes of four targets, whose loads are on their way at once; eight threads to a target's block of 128 dimensions.
__global__ void __launch_bounds__(256) map_stage_kernel(const __grid_constant__ Map P, const int nby, const int nbv)
{
    constexpr int PER = 4;
    const int c16 = threadIdx.x & 7, r0 = threadIdx.x >> 3, b0 = blockIdx.x, t = blockIdx.y, w = blockIdx.z;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");               // (which waits for all of this grid's writes)
    const int tiles = gridDim.y, len = map_length(P, w);
    if (t * 128 >= len) return;                                                // (a tile that no one reads)
    const bool value = b0 >= nby;
    const int b = value ? b0 - nby : b0;
    const Cloud8 &cl = value ? P.v : P.y;
    uint4 codes[PER];
    uint32_t e[PER];
    double g[PER];
    float norm[PER];
#pragma unroll
    for (int a = 0; a < PER; ++a) {
        const size_t at = (size_t)w * P.m + min(t * 128 + r0 + 32 * a, len - 1);
        e[a] = cl.scales[at * cl.sb + b];
        codes[a] = make_uint4(0u, 0u, 0u, 0u);
        if (b * 128 + c16 * 16 < cl.cb) codes[a] = *reinterpret_cast<const uint4 *>(cl.codes + at * cl.cb + b * 128 + c16 * 16);
        g[a] = P.g ? P.g[at] : 0.0;
        norm[a] = P.y.norms[at];
    }
    unsigned char *dst0 = (value ? P.staged_v : P.staged_y) + (((size_t)w * tiles + t) * (value ? nbv : nby) + b) * MT_BLOCK + (c16 >> 2) * MT_CHUNK;
    const int c0 = 2 * (c16 & 3);
#pragma unroll
    for (int a = 0; a < PER; ++a) {
        const int r = r0 + 32 * a;
        const bool hidden = t * 128 + r >= len || g[a] == -INFINITY, masked = hidden || norm[a] == INFINITY;
        if (b0 == 0 && c16 == 0) P.terms[((size_t)w * tiles + t) * 128 + r] = hidden ? -INFINITY : map_term(map_scale(P, w), g[a], norm[a]);
        // what codes are multiplied by, 2^(120 + E), in one step where bf16 holds it; masked targets and their values are zeros
        const uint32_t e1 = min(e[a], 134u);
        uint32_t f = masked ? 0u : e[a] == 255u ? 0x7fffu : (e1 + 120u) << 7;
        f |= f << 16;
        const uint32_t wd[4] = {codes[a].x, codes[a].y, codes[a].z, codes[a].w};
        uint32_t h[8];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            h[2 * x] = mul_bf16x2(codes_bf16(__byte_perm(wd[x], 0u, 0x1404)), f);
            h[2 * x + 1] = mul_bf16x2(codes_bf16(__byte_perm(wd[x], 0u, 0x3424)), f);
        }
        if (!masked && e[a] > 134u && e[a] != 255u) {
            uint32_t more = (e[a] - 134u + 127u) << 7;
            more |= more << 16;
#pragma unroll
            for (int x = 0; x < 8; ++x) h[x] = mul_bf16x2(h[x], more);
        }
        unsigned char *dst = dst0 + r * 128;
        *reinterpret_cast<uint4 *>(dst + ((c0 ^ (r & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4 *>(dst + (((c0 + 1) ^ (r & 7)) << 4)) = make_uint4(h[4], h[5], h[6], h[7]);
    }
}

// PAIR: two blocks of a cluster share what they read, half of the targets (scores) or of the dimensions (images) of a stage each; the first issues
// the instructions of both, on 256 queries.  LONG: a part may have more tiles than MT_CHAIN.  (A kernel of its own: the softmax has no registers left for what that
// takes; 64 x 1024 x 1024 x 512 would take 1 % longer.  Parts that are long take 2 to 3 % longer for it.)
template <int DVC, bool PAIR, bool LONG>
__global__ void __launch_bounds__(MT_THREADS, 1) map_tiles_kernel(const __grid_constant__ CUtensorMap tmx, const __grid_constant__ CUtensorMap tmy,
                                                                  const __grid_constant__ CUtensorMap tmv, const __grid_constant__ Map P, const int nrt,
                                                                  const int stages, const int lane_tiles, const int tma_x, const int wave)
{
    constexpr uint32_t STAGE = PAIR ? MT_BLOCK / 2 : MT_BLOCK;
    extern __shared__ __align__(1024) unsigned char smem_dyn[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rt = blockIdx.x % nrt, z = blockIdx.x / nrt, split = blockIdx.y, w = blockIdx.z;
    const uint32_t rank = PAIR ? blockIdx.x & 1u : 0u;
    const int i0 = rt * 128, dv0 = z * DVC;
    const int nkc = (P.d + 63) / 64, nby = (P.d + 127) / 128, nbv = (min(DVC, P.dv - dv0) + 127) / 128;

    // shared memory: the queries' chunks, the ring, and what is small
    const uint32_t base = smem_u32(smem_dyn), sX = base, sR = base + (uint32_t)nkc * MT_CHUNK;
    unsigned char *misc = smem_dyn + (size_t)nkc * MT_CHUNK + (size_t)stages * STAGE;
    float *terms = reinterpret_cast<float *>(misc);                        // [2][128]
    float *tops = terms + 256;                                             // [2][128]: halves' maxima, and their sums at the end
    unsigned long long *bars = reinterpret_cast<unsigned long long *>(tops + 256);
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(bars + 32);
    float *refs = reinterpret_cast<float *>(bars + 36);                    // [128]: what the images in P.sums are against
    int *abort_flag = reinterpret_cast<int *>(tmem_holder + 1), *mine = abort_flag + 1;      // mine: the first of this part's tiles, among all lanes', and how many
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    constexpr int FULL = 0, EMPTY = MT_MAX_STAGES, SFULL = 2 * MT_MAX_STAGES, PFULL = SFULL + 2, ODONE = PFULL + 2, TFULL = ODONE + 1, TEMPTY = TFULL + 2,
                  LAST = TEMPTY + 2, XFULL = LAST + 1;
    static_assert(XFULL < 32, "barriers");

    const int len = map_length(P, w), tiles = (len + 127) / 128;
    const int t0 = (int)((long long)tiles * split / P.splits), t1 = (int)((long long)tiles * (split + 1) / P.splits), nt = t1 - t0;
    if (tid == 0) {
        for (int s = 0; s < stages; ++s) { mbar_init(bar(FULL + s), 1); mbar_init(bar(EMPTY + s), 1); }
        for (int b = 0; b < 2; ++b) {
            mbar_init(bar(SFULL + b), 1);
            mbar_init(bar(PFULL + b), PAIR ? 2 * MT_SOFT : MT_SOFT);
            mbar_init(bar(TFULL + b), 1);
            mbar_init(bar(TEMPTY + b), MT_SOFT);
        }
        mbar_init(bar(ODONE), 1);
        mbar_init(bar(LAST), 1);
        mbar_init(bar(XFULL), 1);
        mine[0] = w * lane_tiles + t0;                                     // (here, as they take registers of the softmax else, which has none left)
        mine[1] = nt;
        *abort_flag = (base & 1023u) ? 1 : 0;                              // (the swizzle counts from 1024-byte boundaries)
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MT_MMA) {
        if constexpr (!PAIR) tc_alloc<512>(tmem_holder);
        else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_holder)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    // the queries: by TMA (below), or where their rows are no whole number of 16 bytes by the threads, one value after the other
    if (!tma_x)
        for (int i = tid; i < 128 * 8 * nkc; i += MT_THREADS) {
            const int r = i / (8 * nkc), ch = i % (8 * nkc), k0 = 8 * ch;
            uint32_t v[4] = {0u, 0u, 0u, 0u};
            if (i0 + r < P.n) {
                const uint16_t *src = P.x + ((size_t)w * P.n + i0 + r) * P.d + k0;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (k0 + e < P.d) v[e / 2] |= (uint32_t)src[e] << (16 * (e & 1));
            }
            *reinterpret_cast<uint4 *>(smem_dyn + (size_t)(ch / 8) * MT_CHUNK + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
        }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();                                // both blocks' barriers are there, and their queries
    tc_fence_after();
    const uint32_t tmem = *tmem_holder, tO = tmem + 256;
    volatile int *ab = abort_flag;
    const double k = map_scale(P, w);

    if (warp < MT_SOFT) {
        const int half = warp >> 2, q = (warp & 3) * 32 + lane;            // query; half of a tile's targets and of the image's dimensions
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const float kx = (float)(2.0 * k);
        const u64 k2 = pack2(kx, kx);
        float ref = -INFINITY;
        double sum = 0.0;
        bool ok = *ab == 0;
        const bool starts = ok;
        const bool want_xx = P.lse && z == 0 && P.splits == 1;
        double xx = 0.0;
        // images in P.sums: a block's lie together, a thread's 256 floats apart
        auto sums_of = [&] {
            return P.sums + (blockIdx.x + (size_t)gridDim.x * (blockIdx.y + (size_t)gridDim.y * blockIdx.z)) * (128 * DVC) + tid;
        };
        // ... which are multiplied by this when the reference is another
        auto since = [&](float was) { return was == -INFINITY ? 0.f : ex2_fast(was - ref); };
        if (LONG && half == 0) refs[q] = -INFINITY;
        for (int t = 0; t < nt && starts; ++t) {
            const int b = t & 1;
            const uint32_t ph = (uint32_t)(t >> 1) & 1u;
            if (LONG && t && t % MT_CHAIN == 0) {
                // what has been added up in tensor memory joins the rest in fp32; the instructions begin anew.  (One phase after the other: see the end.)
                ok = ok && mbar_wait(bar(ODONE), (uint32_t)(t - 2) & 1u, ab) && mbar_wait(bar(ODONE), (uint32_t)(t - 1) & 1u, ab);
                ok = __all_sync(0xffffffffu, ok);
                tc_fence_after();
                const float was = refs[q], fac = since(was);
                asm volatile("bar.sync %0, 64;" ::"r"(1 + (warp & 3)) : "memory");
                if (half == 0) refs[q] = ref;
                float *at = sums_of();
                if (ok)
#pragma unroll 1
                    for (int c = 0; c < DVC / 2; c += 16, at += 16 * 32 * MT_SOFT) {
                        uint32_t o[16];
                        float rest[16];                                    // (all loads before the first store)
                        tc_ld16_issue(tO + lanes + half * (DVC / 2) + c, o);
#pragma unroll
                        for (int i = 0; i < 16; ++i) rest[i] = t > MT_CHAIN ? at[i * 32 * MT_SOFT] : 0.f;
                        tc_ld16_wait(o);
#pragma unroll
                        for (int i = 0; i < 16; ++i) at[i * 32 * MT_SOFT] = fmaf(rest[i], fac, __uint_as_float(o[i]));
                    }
            }
            ok = ok && mbar_wait(bar(TFULL + b), ph, ab) && mbar_wait(bar(SFULL + b), ph, ab);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            const uint32_t sS = tmem + lanes + 128 * b;
            float top = -INFINITY;
            u64 v[2][16];
            if (ok) {
                uint32_t r[2][32];
                tc_ld32_issue(sS + 64 * half, r[0]);
                tc_ld32_issue(sS + 64 * half + 32, r[1]);
                tc_ld_wait(r[0]);
                tc_ld_wait(r[1]);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 c = *reinterpret_cast<const float4 *>(terms + 128 * b + 64 * half + 32 * h + i);
                        v[h][i / 2] = fma2(pack2(__uint_as_float(r[h][i]), __uint_as_float(r[h][i + 1])), k2, pack2(c.x, c.y));
                        v[h][i / 2 + 1] = fma2(pack2(__uint_as_float(r[h][i + 2]), __uint_as_float(r[h][i + 3])), k2, pack2(c.z, c.w));
                        float a0, a1, a2, a3;
                        unpack2(v[h][i / 2], a0, a1);
                        unpack2(v[h][i / 2 + 1], a2, a3);
                        top = fmaxf(fmaxf(top, fmaxf(a0, a1)), fmaxf(a2, a3));
                    }
            }
            tops[128 * half + q] = top;
            // both halves have read S (its place is P's next) and know the query's maximum, and whether either has given up
            ok = all_of<64>(ok, 1 + (warp & 3));
            if (!ok) break;
            if (lane == 0) mbar_arrive(bar(TEMPTY + b));
            top = fmaxf(top, tops[128 * (1 - half) + q]);
            // (read before either half writes the next tile's)
            asm volatile("bar.sync %0, 64;" ::"r"(1 + (warp & 3)) : "memory");
            float fac = 1.f;
            if (top > ref + MT_SLACK || (ref == -INFINITY && top > -INFINITY)) {
                const float up = ceilf(top);
                fac = ex2_fast(ref - up);
                ref = up;
            }
            const bool raise = __any_sync(0xffffffffu, fac != 1.f);
            if (raise) {
                sum *= (double)fac;
                if (t > 0) {
                    // (O of the tile before the last is there: S of this tile was issued after it)
                    // (where that wait runs out the halves part only at the next tile's barrier)
                    ok = mbar_wait(bar(ODONE), (uint32_t)(t - 1) & 1u, ab);
                    ok = __all_sync(0xffffffffu, ok);
                    tc_fence_after();
                    for (int c = 0; c < DVC / 2; c += 32) {
                        const uint32_t at = tO + lanes + half * (DVC / 2) + c;
                        uint32_t o[32];
                        tc_ld32_issue(at, o);
                        tc_ld_wait(o);
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * fac);
                        tc_st32_issue(at, o);
                    }
                }
            }
            const float at = ref == -INFINITY ? 0.f : ref;
            const u64 at2 = pack2(-at, -at);
            u64 acc[2] = {0ull, 0ull};
            uint32_t p[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                float a, c;
                unpack2(add2(v[i / 16][i % 16], at2), a, c);
                a = ex2_fast(a);
                c = ex2_fast(c);
                acc[i & 1] = add2(acc[i & 1], pack2(a, c));
                p[i] = bf16_pair(a, c);
            }
            tc_st32_issue(sS + 32 * half, p);
            float a, c;
            unpack2(add2(acc[0], acc[1]), a, c);
            sum += (double)(a + c);
            tc_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                // (what the instructions read of this thread's is in tensor memory, ordered by the fence above; a release of all else to the cluster
                // takes as long as half a tile)
                if constexpr (PAIR)
                    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_block(bar(PFULL + b), 0)) : "memory");
                else mbar_arrive(bar(PFULL + b));
            }
            if (t == 0 && want_xx) {
                // |x|^2 of this half of the query's dimensions, while there is time: eight sums in fp32 of a value of every eight, added up in double every 64.
                // (The queries are there: scores were made of them.)
                for (int c = half; c < nkc; c += 2) {
                    float part[8];
    #pragma unroll
                    for (int e = 0; e < 8; ++e) part[e] = 0.f;
    #pragma unroll
                    for (int ch = 0; ch < 8; ++ch) {
                        const uint4 u = *reinterpret_cast<const uint4 *>(smem_dyn + (size_t)c * MT_CHUNK + q * 128 + ((ch ^ (q & 7)) << 4));
                        const uint32_t h[4] = {u.x, u.y, u.z, u.w};
    #pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float lo = __uint_as_float(h[e] << 16), hi = __uint_as_float(h[e] & 0xffff0000u);
                            part[2 * e] = fmaf(lo, lo, part[2 * e]);
                            part[2 * e + 1] = fmaf(hi, hi, part[2 * e + 1]);
                        }
                    }
                    xx += (double)(((part[0] + part[1]) + (part[2] + part[3])) + ((part[4] + part[5]) + (part[6] + part[7])));
                }
            }
        }
        if (ok && nt > 0) {
            // (one phase after the other: the wait for a phase is over as well while the one before it has yet to end)
            if (nt > 1) ok = mbar_wait(bar(ODONE), (uint32_t)(nt - 2) & 1u, ab);
            ok = ok && mbar_wait(bar(ODONE), (uint32_t)(nt - 1) & 1u, ab);
            tc_fence_after();
        }
        ok = __all_sync(0xffffffffu, ok);
        const float nan = __uint_as_float(0x7fffffffu);
        float total = ok ? (float)sum : nan;
        // Where a query or eps is no number, scores of masked targets are NaN like others: a sum that is NaN is one of nothing if no target of this part counts.
        // (The terms once more, for such sums alone: a comparison in the softmax takes one percent of the whole.)
        if (!all_of<32 * MT_SOFT>(total == total, 5)) {
            asm volatile("griddepcontrol.wait;" ::: "memory");
            const volatile int *own = mine;
            const float *term = P.terms + (size_t)own[0] * 128;
            const int count = own[1] * 128;
            bool any = !ok;
            for (int i = tid; i < count; i += 32 * MT_SOFT) any |= term[i] != -INFINITY;
            if (all_of<32 * MT_SOFT>(!any, 5)) { total = 0.f; ref = -INFINITY; }
        }
        // (both halves leave the loop at the same tile, after they have read its maxima, or neither has)
        tops[128 * half + q] = total;
        asm volatile("bar.sync %0, 64;" ::"r"(1 + (warp & 3)) : "memory");
        total += tops[128 * (1 - half) + q];
        const bool some = __any_sync(0xffffffffu, total != 0.f);          // (else there are no images)
        const bool live = i0 + q < P.n;
        const size_t row = (size_t)w * P.n + i0 + (live ? q : 0);
        const float inv = P.splits > 1 ? (total == total ? 1.f : nan) : total == 0.f ? 0.f : 1.f / total;
        // images by way of shared memory, which queries and stages need no more, so that rows are written whole
        const bool whole = all_of<32 * MT_SOFT>(ok, 5) && P.splits == 1 && P.dv % 8 == 0 && (uintptr_t)P.out % 16 == 0;
        constexpr int ROW = 2 * DVC;                                       // bytes
        for (int c = 0; c < DVC / 2; c += 32) {
            const int dim = dv0 + half * (DVC / 2) + c;
            if (dim >= P.dv) break;
            uint32_t o[32];
            if (some) {
                tc_ld32_issue(tO + lanes + half * (DVC / 2) + c, o);
                tc_ld_wait(o);
            } else
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = 0u;
            if (LONG && some && nt > MT_CHAIN) {
                const float fac = since(refs[q]);
                const float *at = sums_of() + c * 32 * MT_SOFT;
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(fmaf(at[i * 32 * MT_SOFT], fac, __uint_as_float(o[i])));
            }
            if (P.splits > 1) {
                float *dst = P.part_out + (row * P.splits + split) * P.dv + dim;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (live && dim + i < P.dv) dst[i] = __uint_as_float(o[i]) * inv;
                continue;
            }
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
                uint32_t h[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = bf16_pair(__uint_as_float(o[i + 2 * e]) * inv, __uint_as_float(o[i + 2 * e + 1]) * inv);
                if (whole) {
                    const int ch = (half * (DVC / 2) + c + i) / 8;
                    *reinterpret_cast<uint4 *>(smem_dyn + q * ROW + ((ch ^ (q & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
                } else if (live)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (dim + i + e < P.dv) P.out[row * P.dv + dim + i + e] = (uint16_t)(h[e / 2] >> (16 * (e & 1)));
            }
        }
        if (P.splits == 1 && P.lse && z == 0) {
            // (the sums have been read: the barrier of all eight warps came after)
            double *halves = reinterpret_cast<double *>(terms);
            if (half) halves[q] = xx;
            asm volatile("bar.sync %0, 64;" ::"r"(1 + (warp & 3)) : "memory");
            if (live && half == 0) P.lse[row] = map_lse(ref, total, k, xx + halves[q]);
        }
        if (P.splits > 1 && live && half == 0 && z == 0) reinterpret_cast<float2 *>(P.part_ml)[row * P.splits + split] = make_float2(ref, total);
        if (whole) {
            asm volatile("bar.sync 5, %0;" ::"n"(32 * MT_SOFT) : "memory");
            constexpr int PER = ROW / 16;                                  // 16-byte pieces of a row
            for (int i = tid; i < 128 * PER; i += 32 * MT_SOFT) {
                const int r = i / PER, ch = i % PER, dim = dv0 + 8 * ch;
                if (i0 + r < P.n && dim < P.dv)
                    *reinterpret_cast<uint4 *>(P.out + ((size_t)w * P.n + i0 + r) * P.dv + dim) =
                        *reinterpret_cast<const uint4 *>(smem_dyn + r * ROW + ((ch ^ (r & 7)) << 4));
            }
        }
    } else if (warp == MT_LOAD) {
        if (lane == 0) {
            const long long y0 = ((long long)w * lane_tiles + t0) * nby, all_v = (P.dv + 127) / 128;
            const long long v0 = ((long long)w * lane_tiles + t0) * all_v + dv0 / 128;     // blocks of 128 targets by 128 dimensions
            const float *term = P.terms + ((size_t)w * lane_tiles + t0) * 128;
            bool ok = *ab == 0;
            // (a stage's number and its phase are counted, not divided out: a division is longer than a stage's instructions take to issue)
            int i = 0, s = 0;
            uint32_t ph = 0;
            auto stage = [&](bool value, long long block) {
                if (!(ok = mbar_wait(bar(EMPTY + s), ph ^ 1u, ab))) return;
                const uint32_t dst = sR + s * STAGE;
                if constexpr (!PAIR) {
                    mbar_expect_tx(bar(FULL + s), STAGE);
                    bulk_load(dst, (value ? P.staged_v : P.staged_y) + (size_t)block * MT_BLOCK, STAGE, bar(FULL + s));
                } else {
                    // scores: both halves of 64 dimensions of this block's 64 targets; images: all targets of its 64 dimensions
                    if (rank == 0) mbar_expect_tx(bar(FULL + s), 2 * STAGE);
                    const uint32_t full = in_block(bar(FULL + s), 0);
                    const int row = (int)(block * 256) + (value ? 128 : 64) * (int)rank;
                    load_rows(dst, value ? &tmv : &tmy, row, full);
                    load_rows(dst + STAGE / 2, value ? &tmv : &tmy, row + (value ? 64 : 128), full);
                }
                ++i;
                if (++s == stages) { s = 0; ph ^= 1u; }
            };
            int terms_issued = 0;
            if (tma_x && ok && nt > 0) {
                if (rank == 0) mbar_expect_tx(bar(XFULL), (PAIR ? 2 : 1) * nkc * MT_CHUNK);
                for (int c = 0; c < nkc; ++c) load_queries<PAIR>(sX + c * MT_CHUNK, &tmx, 64 * c, i0, w, PAIR ? in_block(bar(XFULL), 0) : bar(XFULL));
            }
            // the queries of the block that follows on this SM, about, into L2
            if (tma_x) {
                const long long later = (long long)blockIdx.x + (long long)gridDim.x * ((long long)blockIdx.y + (long long)gridDim.y * blockIdx.z) + wave;
                const long long lw = later / ((long long)gridDim.x * gridDim.y);
                const int lrt = (int)(later % gridDim.x) % nrt;
                if (lw < P.W)
                    for (int c = 0; c < nkc; ++c)
                        asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];"
                                     ::"l"(reinterpret_cast<uint64_t>(&tmx)), "r"(64 * c), "r"(lrt * 128), "r"((int)lw) : "memory");
            }
            // (the bank as bf16 is there: up to here nothing of it was read)
            asm volatile("griddepcontrol.wait;\n\tfence.proxy.async.global;" ::: "memory");
            // in the order of the matrix instructions: scores of tile t, then images of tile t - 1
            for (int t = 0; t <= nt && nt > 0 && ok; ++t) {
                if (t < nt) {
                    if (!(ok = mbar_wait(bar(TEMPTY + (t & 1)), ((uint32_t)(t >> 1) & 1u) ^ 1u, ab))) break;
                    mbar_expect_tx(bar(TFULL + (t & 1)), 512);
                    bulk_load(smem_u32(terms) + 512 * (t & 1), term + (size_t)t * 128, 512, bar(TFULL + (t & 1)));
                    ++terms_issued;
                    for (int b = 0; b < nby && ok; ++b) stage(false, y0 + (long long)t * nby + b);
                }
                if (t > 0)
                    for (int b = 0; b < nbv && ok; ++b) stage(true, v0 + (t - 1) * all_v + b);
            }
            // nothing may land in shared memory after the block has gone: the last load of every buffer, with a bound of its own.  (A pair's loads
            // are counted at the first block, which waits for both.)
            int unused = 0;
            if (tma_x && nt > 0 && rank == 0) mbar_wait(bar(XFULL), 0, &unused);
            for (int q = max(0, i - stages); q < i && rank == 0; ++q) mbar_wait(bar(FULL + q % stages), (uint32_t)(q / stages) & 1u, &unused);
            // (and no arrival of the other block's instructions)
            for (int q = max(0, i - stages); q < i && PAIR; ++q) mbar_wait(bar(EMPTY + q % stages), (uint32_t)(q / stages) & 1u, &unused);
            for (int q = max(0, terms_issued - 2); q < terms_issued; ++q) mbar_wait(bar(TFULL + (q & 1)), (uint32_t)(q >> 1) & 1u, &unused);
        }
    } else {
        // (the whole warp walks through the stages, so that descriptors are uniform; one thread issues)
        if (rank == 0) {
            bool ok = *ab == 0;
            int s = 0;
            uint32_t ph = 0;
            auto next = [&] { if (++s == stages) { s = 0; ph ^= 1u; } };
            const uint64_t x0 = tc_desc(sX), r0 = tc_desc(sR), v0 = desc_columns(sR);     // (an address counts units of 16 bytes)
            if (tma_x && nt > 0 && ok) ok = __all_sync(0xffffffffu, mbar_wait(bar(XFULL), 0, ab));
            tc_fence_after();
            for (int t = 0; t <= nt && nt > 0 && ok; ++t) {
                if (t < nt)
                    for (int b = 0; b < nby; ++b, next()) {
                        if (!(ok = __all_sync(0xffffffffu, mbar_wait(bar(FULL + s), ph, ab)))) break;
                        tc_fence_after();
                        const uint64_t xd = x0 + (uint64_t)(b * 2 * (int)(MT_CHUNK >> 4)), yd = r0 + (uint64_t)(s * (int)(STAGE >> 4));
                        const uint32_t acc = tmem + 128 * (t & 1);
                        const int left = P.d - 128 * b;
                        if (elected()) {
                            mma_smem<PAIR>(acc, xd, yd, b ? 1u : 0u);
                            if (left > 112) {
#pragma unroll
                                for (int q = 1; q < 8; ++q)
                                    mma_smem<PAIR>(acc, xd + (q >> 2) * (MT_CHUNK >> 4) + (q & 3) * 2, yd + (q >> 2) * (STAGE >> 5) + (q & 3) * 2, 1u);
                            } else
                                for (int q = 1; 16 * q < left; ++q)
                                    mma_smem<PAIR>(acc, xd + (q >> 2) * (MT_CHUNK >> 4) + (q & 3) * 2, yd + (q >> 2) * (STAGE >> 5) + (q & 3) * 2, 1u);
                            commit<PAIR>(bar(EMPTY + s));
                            if (b == nby - 1) commit<PAIR>(bar(SFULL + (t & 1)));
                        }
                        __syncwarp();
                    }
                if (t == 0 || !ok) continue;
                const int u = t - 1;
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(bar(PFULL + (u & 1)), (uint32_t)(u >> 1) & 1u, ab)))) break;
                tc_fence_after();
                for (int b = 0; b < nbv; ++b, next()) {
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait(bar(FULL + s), ph, ab)))) break;
                    tc_fence_after();
                    const uint64_t vd = v0 + (uint64_t)(s * (int)(STAGE >> 4));
                    const uint32_t out = tO + 128 * b, weights = tmem + 128 * (u & 1);
                    if (elected()) {
                        mma_tmem<PAIR>(out, weights, vd, (LONG ? u % MT_CHAIN : u) ? 1u : 0u);
#pragma unroll
                        for (int q = 1; q < 8; ++q) mma_tmem<PAIR>(out, weights + 8 * q, vd + q * (2048 >> 4), 1u);
                        commit<PAIR>(bar(EMPTY + s));
                        if (b == nbv - 1) commit<PAIR>(bar(ODONE));
                    }
                    __syncwarp();
                }
            }
            // what was issued is over before tensor memory is given back
            if (elected()) {
                commit<PAIR>(bar(LAST), 1);
                int unused = 0;
                mbar_wait(bar(LAST), 0, &unused);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    // (neither block of a pair goes while the other's instructions and loads may still use its memory)
    if constexpr (PAIR) cluster_sync_all();
    if (warp == MT_MMA) {
        if constexpr (!PAIR) tc_dealloc<512>(tmem);
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <int DVC, bool PAIR, bool LONG>
skb_status launch(const CUtensorMap &tx, const CUtensorMap &ty, const CUtensorMap &tv, const Map &P, int tma_x, int sms, cudaStream_t st)
{
    constexpr int stage = PAIR ? (int)MT_BLOCK / 2 : (int)MT_BLOCK;
    const int nkc = (P.d + 63) / 64, blocks = (P.n + 127) / 128, nrt = PAIR ? (blocks + 1) / 2 * 2 : blocks, nz = (P.dv + DVC - 1) / DVC;
    const int stages = min(MT_MAX_STAGES, (MAP_TILES_SMEM - (int)MT_MISC - nkc * (int)MT_CHUNK) / stage);
    const int smem = nkc * (int)MT_CHUNK + stages * stage + (int)MT_MISC;
    cudaFuncSetAttribute(map_tiles_kernel<DVC, PAIR, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(nrt * nz, P.splits, P.W);
    cfg.blockDim = dim3(MT_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    // (it may start before the bank is staged, and waits for that)
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = PAIR ? 2 : 1;
    cudaLaunchKernelEx(&cfg, map_tiles_kernel<DVC, PAIR, LONG>, tx, ty, tv, P, nrt, stages, (P.m + 127) / 128, tma_x, sms);
    return op_launched("map");
}

}  // namespace

// rows of 128 queries, and columns of values, that a launch's blocks take
static int row_blocks(int n) { return n > 128 ? (n + 255) / 256 * 2 : 1; }
static int value_depth(int dv) { return dv <= 128 ? 128 : (dv + 255) / 256 * 256; }

size_t map_staged_bytes(int W, int n, int m, int d, int dv, bool own_values, int splits)
{
    const int lane_tiles = (m + 127) / 128;
    const size_t tiles = (size_t)W * lane_tiles;
    const size_t sums = lane_tiles > MT_CHAIN ? (size_t)W * splits * row_blocks(n) * 128 * value_depth(dv) * sizeof(float) : 0;
    return tiles * 512 + tiles * MT_BLOCK * ((d + 127) / 128 + (own_values ? (dv + 127) / 128 : 0)) + sums;
}

skb_status launch_map_tiles(Map &P, void *room, int sms, cudaStream_t st)
{
    const int tiles = (P.m + 127) / 128, nby = (P.d + 127) / 128, nbv = P.own_values ? (P.dv + 127) / 128 : 0;
    P.staged_y = (unsigned char *)room;
    P.staged_v = P.own_values ? P.staged_y + (size_t)P.W * tiles * nby * MT_BLOCK : P.staged_y;
    P.terms = (float *)(P.staged_y + (size_t)P.W * tiles * (nby + nbv) * MT_BLOCK);
    P.sums = tiles > MT_CHAIN ? P.terms + (size_t)P.W * tiles * 128 : nullptr;
    map_stage_kernel<<<dim3(nby + nbv, tiles, P.W), 256, 0, st>>>(P, nby, nbv);
    const skb_status rc = op_launched("map");
    if (rc != SKB_OK) return rc;
    const bool pair = P.n > 128;
    CUtensorMap tx = {}, ty = {}, tv = {};
    const int tma_x = P.d % 8 == 0 && (uintptr_t)P.x % 16 == 0;
    if ((tma_x && !queries_map(&tx, P.x, P.d, P.n, P.W)) ||
        (pair && (!staged_map(&ty, P.staged_y, (size_t)P.W * tiles * nby * 256) ||
                 !staged_map(&tv, P.staged_v, (size_t)P.W * tiles * (P.own_values ? nbv : nby) * 256))))
        return op_fail(SKB_ERR_CUDA, "cuTensorMapEncodeTiled failed");
    const bool longer = (tiles + P.splits - 1) / P.splits > MT_CHAIN;
    const auto by_depth = [&](auto two, auto chained) {
        return P.dv <= 128 ? launch<128, two.value, chained.value>(tx, ty, tv, P, tma_x, sms, st) : launch<256, two.value, chained.value>(tx, ty, tv, P, tma_x, sms, st);
    };
    const std::true_type yes;
    const std::false_type no;
    if (pair) return longer ? by_depth(yes, yes) : by_depth(yes, no);
    return longer ? by_depth(no, yes) : by_depth(no, no);
}

}  // namespace skb
