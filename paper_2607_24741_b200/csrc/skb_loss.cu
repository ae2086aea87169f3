// The loss of scores against the rows of a coupling, and its gradient: distillation of the entries that a teacher names.
//
// Row i has scores s_ij, p = softmax(s / T), and k named entries (draws from the plan's row, or its top entries with logits t),
//      q = softmax(t / T) over the named entries,   loss_i = sum_k q_k (log q_k - log p_{j(k)}),
//      d loss_i / d s_ij = (p_ij - sum of q_k over the k with j(k) = j) / T.
//
// One pass: a row is read once, 16 bytes a thread and vector, and stays in registers (up to 64 scores of bf16 or 32 of fp32 a
// thread, raw) until its maximum and sum are known; then the gradient is written.  So memory bounds it, and the latencies of what a row
// needs besides: 65536 rows of 1024 in bf16 take 47 us for 270 MB (87 % of the measured copy rate; 52 for a call by itself; 28 without the
// gradient), of 64 12.  Exponentials are taken against the
// thread's own maximum for the sum; short rows keep them, others take them again against the row's: that is one barrier a row instead of two, and no fp32
// copies in registers.  What a row is given goes by its length (launch_by_length): a quarter of a warp, half of one, a warp, four, eight or 16 warps, or a cluster of up to eight blocks, whose
// maxima and sums meet in distributed shared memory; long rows, a device full of them, stay in shared memory (loss_long_kernel); rows longer than what a cluster's registers hold are read twice, the second time from L2 (a row
// is at most 1 MB).  A row is reduced in a fixed order, so results do not change from call to call.
//
// The named entries, a thread to each, are fetched before the row and their softmax is made while it is on its way.  Their gradients are written after
// all others of the row, by the first of the entries that name a column, which adds up the q of all that do: no atomics, any entry may be named
// any number of times.
#include <cuda_runtime.h>
#include <string>

#include "skb_f32x2.cuh"
#include "skb_operators.h"
#include "skb_tmem.cuh"

namespace skb {
namespace {

constexpr int LS_MAX_K = 256;

struct Loss {
    const void *scores;
    const int *index;
    const float *logits, *weight;
    float *loss;
    void *grad;
    long long rows, ld, ldg;                  // ld, ldg: elements from row to row
    int m, k;
    float inv_t, c;                           // 1 / T and log2(e) / T
};

// two scores of a vector
template <bool BF16> __device__ __forceinline__ u64 two(const uint4 &v, int i)
{
    if constexpr (BF16) {
        const uint32_t w = i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
        return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    } else
        return i == 0 ? pack2(__uint_as_float(v.x), __uint_as_float(v.y)) : pack2(__uint_as_float(v.z), __uint_as_float(v.w));
}
// the largest score of a vector; NaN counts as none
template <bool BF16> __device__ __forceinline__ float largest(const uint4 &v)
{
    if constexpr (BF16) {
        uint32_t a, b;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
        asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
        return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
    } else
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
}
__device__ __forceinline__ u64 mul2(u64 a, u64 b)
{
    u64 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// 2^((s - at) c) of two scores: the difference first, so that its rounding is of the distance, however large scores are
__device__ __forceinline__ u64 exponentials(u64 s, u64 at2, u64 c2)
{
    float a, b;
    unpack2(mul2(sub2(s, at2), c2), a, b);
    return pack2(ex2_fast(a), ex2_fast(b));
}
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }
// (maximum, sum of exponentials against it), both of none: (-inf, 0)
struct __align__(8) Part {                   // (written to other blocks in one 8-byte store)
    float m, s;
};
// ... of COUNT threads next to each other (the others of a warp: of none)
template <int COUNT> __device__ __forceinline__ Part join(Part p, float c)
{
    const float m = warp_max(p.m), at = finite_max(m);
    // (a sum beside a maximum of minus infinity is 0, or NaN, which stays)
    float s = p.s * ex2_fast((p.m - at) * c);
#pragma unroll
    for (int off = COUNT / 2; off; off /= 2) s += __shfl_xor_sync(0xffffffffu, s, off);
    return {m, s};
}
// the largest of COUNT threads next to each other, and a join of as many, where a warp has several groups of them
template <int COUNT> __device__ __forceinline__ float group_max(float v)
{
    if constexpr (COUNT >= 32) return warp_max(v);
    else {
#pragma unroll
        for (int off = COUNT / 2; off; off /= 2) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
        return v;
    }
}
template <int COUNT> __device__ __forceinline__ Part group_join(Part p, float c)
{
    if constexpr (COUNT >= 32) return join<32>(p, c);
    else {
        const float m = group_max<COUNT>(p.m);
        float s = p.s * ex2_fast((p.m - finite_max(m)) * c);
#pragma unroll
        for (int off = COUNT / 2; off; off /= 2) s += __shfl_xor_sync(0xffffffffu, s, off);
        return {m, s};
    }
}
__device__ __forceinline__ Part join(Part a, Part b, float c)
{
    const float m = fmaxf(a.m, b.m), at = finite_max(m);
    return {m, a.s * ex2_fast((a.m - at) * c) + b.s * ex2_fast((b.m - at) * c)};
}

// TPR threads of each of C blocks to a row, V vectors in each thread's registers; V = 0: the row is read twice.  EVEN: rows and gradients are whole vectors.
template <bool BF16, int TPR, int V, int C, bool EVEN>
__global__ void __launch_bounds__(TPR <= 256 ? 256 : TPR, TPR <= 256 ? 4 : 2) loss_kernel(const __grid_constant__ Loss P)
{
    constexpr int THREADS = TPR <= 256 ? 256 : TPR, GROUPS = THREADS / TPR, WARPS = TPR < 32 ? 1 : TPR / 32, SPAN = TPR < 32 ? TPR : 32;
    constexpr int E = BF16 ? 8 : 4;
    using T = typename std::conditional<BF16, uint16_t, uint32_t>::type;
    extern __shared__ float s_entries[];                          // [GROUPS][4][k]: index, q, log q, score
    __shared__ float s_loss[GROUPS][WARPS];
    __shared__ Part s_part[GROUPS][WARPS], s_teach[GROUPS][WARPS], s_rank[C];
    const int tid = threadIdx.x, group = tid / TPR, t = tid % TPR, lane = tid & 31, warp = t >> 5;
    const int rank = C > 1 ? (int)(blockIdx.x % C) : 0;
    const long long row_at = (long long)(blockIdx.x / C) * GROUPS + group;
    // whole groups go: barriers below are a group's.  (Those of a part of a warp stay for its shuffles, and write nothing.)
    if (TPR >= 32 && row_at >= P.rows) return;
    const bool there = TPR >= 32 || row_at < P.rows;
    const long long row = there ? row_at : P.rows - 1;
    int *s_index = reinterpret_cast<int *>(s_entries) + (size_t)group * 4 * P.k;
    float *s_q = reinterpret_cast<float *>(s_index) + P.k, *s_log = s_q + P.k, *s_score = s_log + P.k;
    auto group_sync = [&] {
        if constexpr (TPR <= 32) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(TPR) : "memory");
    };
    // (a block's shared memory may be written by another of its cluster once it has started)
    if constexpr (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const T *src = (const T *)P.scores + (size_t)row * P.ld;
    const int head = EVEN ? 0 : (int)((uintptr_t)src % 16 / sizeof(T)), end = head + P.m;      // the row, in elements from a 16-byte boundary on
    const T *base = src - head;
    const int nvec = (end + E - 1) / E;
    const uint4 nothing = BF16 ? make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u)
                               : make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u);           // minus infinity
    auto load = [&](int j) {
        if (EVEN || (j * E >= head && (j + 1) * E <= end)) return *reinterpret_cast<const uint4 *>(base + (size_t)j * E);
        uint32_t w[4] = {nothing.x, nothing.y, nothing.z, nothing.w};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int at = j * E + e;
            if (at < head || at >= end) continue;
            const uint32_t bits = base[at];
            if (BF16) w[e / 2] = e & 1 ? (w[e / 2] & 0xffffu) | bits << 16 : (w[e / 2] & 0xffff0000u) | bits;
            else w[e] = bits;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    };
    auto score_at = [&](int j) { return BF16 ? __uint_as_float((uint32_t)src[j] << 16) : __uint_as_float((uint32_t)src[j]); };
    // the first entries and the weight are on their way before the row is
    const float weight = P.weight ? P.weight[row] : 1.f;
    int named = -1;
    float logit = 0.f, score = 0.f;                              // of this thread's entry: one to each, a warp's to a row may be more
    if (t < P.k) {
        named = P.index[(size_t)row * P.k + t];
        if (P.logits) logit = P.logits[(size_t)row * P.k + t];
    }
    uint4 held[V ? V : 1];
    if constexpr (V > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int j = (v * C + rank) * TPR + t;
            held[v] = nothing;
            if (j < nvec) held[v] = load(j);
        }
    }
    // the teacher, and the scores that it names, while the row is on its way.  (Logits as they are: as of the scores, differences are taken before anything
    // is multiplied, so that neither a shift of all of them nor their size is felt.)
    Part teach = {-INFINITY, 0.f};
    if (named < 0 || named >= P.m) named = -1;
    const float l0 = named >= 0 ? logit : -INFINITY;
    if (warp * 32 < P.k) {
        if (named >= 0) score = score_at(named);
        teach.m = l0;
        if constexpr (TPR < LS_MAX_K)
            for (int k = t + TPR; k < P.k; k += TPR) {
                int j = P.index[(size_t)row * P.k + k];
                if (j < 0 || j >= P.m) j = -1;
                const float l = j >= 0 ? (P.logits ? P.logits[(size_t)row * P.k + k] : 0.f) : -INFINITY;
                s_index[k] = j;
                s_log[k] = l;
                s_score[k] = j >= 0 ? score_at(j) : 0.f;
                teach.m = fmaxf(teach.m, l);
            }
        teach.m = group_max<SPAN>(teach.m);
        const float at = finite_max(teach.m);
        teach.s = ex2_fast((l0 - at) * P.c);
        // (a thread reads back what it wrote)
        if constexpr (TPR < LS_MAX_K)
            for (int k = t + TPR; k < P.k; k += TPR) teach.s += ex2_fast((s_log[k] - at) * P.c);
#pragma unroll
        for (int off = SPAN / 2; off; off /= 2) teach.s += __shfl_xor_sync(0xffffffffu, teach.s, off);
    }
    // maximum and sum of what this thread has seen
    constexpr bool KEEP = V > 0 && (!BF16 || V <= 4);            // exponentials stay in registers
    Part part = {-INFINITY, 0.f};
    u64 kept[KEEP ? V : 1][E / 2];
    const u64 c2 = pack2(P.c, P.c);
    if constexpr (V > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) part.m = fmaxf(part.m, largest<BF16>(held[v]));
        const u64 at2 = pack2(finite_max(part.m), finite_max(part.m));
        u64 sum[2] = {0ull, 0ull};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                const u64 e = exponentials(two<BF16>(held[v], i), at2, c2);
                if constexpr (KEEP) kept[v][i] = e;
                sum[i & 1] = add2(sum[i & 1], e);
            }
        float a, b;
        unpack2(add2(sum[0], sum[1]), a, b);
        part.s = a + b;
    } else {
        for (int j = rank * TPR + t; j < nvec; j += C * TPR) {
            const uint4 y = load(j);
            Part one = {largest<BF16>(y), 0.f};
            const u64 at2 = pack2(finite_max(one.m), finite_max(one.m));
            u64 sum = 0ull;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) sum = add2(sum, exponentials(two<BF16>(y, i), at2, c2));
            float a, b;
            unpack2(sum, a, b);
            one.s = a + b;
            part = join(part, one, P.c);
        }
    }
    const float own = part.m;
    part = group_join<SPAN>(part, P.c);
    if constexpr (WARPS > 1) {
        if (lane == 0) { s_part[group][warp] = part; s_teach[group][warp] = teach; }
        group_sync();
        teach = join<WARPS>(lane < WARPS ? s_teach[group][lane] : Part{-INFINITY, 0.f}, P.c);
        teach.s = __shfl_sync(0xffffffffu, teach.s, 0);
        part = join<WARPS>(lane < WARPS ? s_part[group][lane] : Part{-INFINITY, 0.f}, P.c);
        part.s = __shfl_sync(0xffffffffu, part.s, 0);
    } else __syncwarp();
    if constexpr (C > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (t < C) {
            uint32_t to;
            const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&s_rank[rank]);
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(mine), "r"(t));
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(part.m), "f"(part.s) : "memory");
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        part = join<C>(lane < C ? s_rank[lane] : Part{-INFINITY, 0.f}, P.c);
        part.s = __shfl_sync(0xffffffffu, part.s, 0);
    }
    const bool live = teach.s != 0.f;                             // (NaN, too)
    const float teach_at = finite_max(teach.m), teach_inv = live ? 1.f / teach.s : 0.f;
    float own_q = 0.f, sum = 0.f;
    if (warp * 32 < P.k) {
        const float log_all = logf(part.s * teach_inv);                // (next to 1 in a confident row, where a fast logarithm is not good)
        // (q log q - q log p)
        auto term = [&](float q, float l, float at) { return q != 0.f ? q * (((l - teach_at) - (at - part.m)) * P.inv_t + log_all) : 0.f; };
        own_q = ex2_fast((l0 - teach_at) * P.c) * teach_inv;
        sum = term(own_q, l0, score);
        if (t < P.k) { s_index[t] = named; s_q[t] = own_q; }
        if constexpr (TPR < LS_MAX_K)
            for (int k = t + TPR; k < P.k; k += TPR) {
                s_q[k] = ex2_fast((s_log[k] - teach_at) * P.c) * teach_inv;
                sum += term(s_q[k], s_log[k], s_score[k]);
            }
        if (rank == 0) {
#pragma unroll
            for (int off = SPAN / 2; off; off /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        }
    }
    if (WARPS > 1 && lane == 0) s_loss[group][warp] = sum;
    // of all warps, in their order
    auto give_loss = [&] {
        if (rank != 0 || t != 0 || !there) return;
        if constexpr (WARPS > 1)
#pragma unroll
            for (int i = 1; i < WARPS; ++i) sum += s_loss[group][i];
        P.loss[row] = live ? sum : 0.f;
    };
    if (!P.grad) {
        group_sync();
        give_loss();
        return;
    }
    const float w = weight * P.inv_t, a = w / part.s;
    T *out = (T *)P.grad + (size_t)row * P.ldg - head;
    const bool wide = EVEN || (uintptr_t)out % 16 == 0;
    // what an exponential is multiplied by: kept ones are against this thread's own maximum.  (That is minus infinity where the thread has seen nothing else: its
    // exponentials, and this, are 0; a row of nothing else has an infinite a and is NaN.)
    const float factor = (KEEP ? ex2_fast((own - finite_max(part.m)) * P.c) : 1.f) * a;
    const u64 at2 = pack2(part.m, part.m), f2 = pack2(factor, factor);
    auto again = [&](const uint4 &y, u64 (&e)[E / 2]) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) e[i] = exponentials(two<BF16>(y, i), at2, c2);
    };
    auto store = [&](int j, const u64 (&e)[E / 2]) {
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            float p, q;
            unpack2(mul2(e[i], f2), p, q);
            if constexpr (BF16) r[i] = bf16_pair(p, q);
            else { r[2 * i] = __float_as_uint(p); r[2 * i + 1] = __float_as_uint(q); }
        }
        if (!live) r[0] = r[1] = r[2] = r[3] = 0u;
        if (EVEN || (wide && j * E >= head && (j + 1) * E <= end)) {
            *reinterpret_cast<uint4 *>(out + (size_t)j * E) = make_uint4(r[0], r[1], r[2], r[3]);
            return;
        }
        if constexpr (!EVEN) {
#pragma unroll
            for (int e1 = 0; e1 < E; ++e1) {
                const int at = j * E + e1;
                if (at >= head && at < end) out[at] = (T)(BF16 ? r[e1 / 2] >> (16 * (e1 & 1)) : r[e1]);
            }
        }
    };
    if constexpr (V > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int j = (v * C + rank) * TPR + t;
            if (j >= nvec || !there) continue;
            if constexpr (!KEEP) {
                // (unpacked anew: the compiler would keep what it unpacked before the barrier, and spill)
                asm volatile("" : "+r"(held[v].x), "+r"(held[v].y), "+r"(held[v].z), "+r"(held[v].w));
                again(held[v], kept[0]);
            }
            store(j, kept[KEEP ? v : 0]);
        }
    } else {
        for (int j = rank * TPR + t; j < nvec; j += C * TPR) {
            again(load(j), kept[0]);
            store(j, kept[0]);
        }
    }
    group_sync();
    give_loss();
    if (!live || warp * 32 >= P.k || !there) return;
    // named entries: each by the first of those that name its column
    if (TPR >= 32 && P.k <= 32) {
        const unsigned alike = __match_any_sync(0xffffffffu, named);
        if (named < 0 || (alike & ((1u << lane) - 1u)) || (C > 1 && (head + named) / E / TPR % C != rank)) return;
        float q = 0.f;
        for (unsigned left = alike; left; left &= left - 1u) q += s_q[__ffs(left) - 1];
        const float g = ex2_fast((score - part.m) * P.c) * a - q * w;
        out[head + named] = BF16 ? (T)bf16_pair(g, 0.f) : (T)__float_as_uint(g);
        return;
    }
    for (int k = t; k < P.k; k += TPR) {
        const int j = k == t ? named : s_index[k];
        if (j < 0 || (C > 1 && (head + j) / E / TPR % C != rank)) continue;
        float q = 0.f;
        bool first = true;
        for (int o = 0; o < P.k; ++o)
            if (s_index[o] == j) {
                first &= o >= k;
                q += s_q[o];
            }
        if (!first) continue;
        const float g = ex2_fast(((k == t ? score : s_score[k]) - part.m) * P.c) * a - q * w;
        out[head + j] = BF16 ? (T)bf16_pair(g, 0.f) : (T)__float_as_uint(g);
    }
}

// Long rows of whole vectors, many of them: a block an SM takes row after row.  A row comes into a ring of 32 KB pieces in shared memory by bulk copies; its
// maximum and sum are made of the pieces as they arrive, the gradient of the same pieces, which go back one by one to the next row's
// copies: reads and writes never stop for the barrier between the two passes.  (In registers of a cluster of four blocks a row of 65536
// in bf16 waits for its slowest block twice: 4096 rows took 249 us, so 211; pieces of 16 KB 231, with 24 warps and 12 KB 252.)
constexpr int LL_WARPS = 16, LL_THREADS = LL_WARPS * 32, LL_PIECE = 32768, LL_PIECES = 6;
template <bool BF16>
__global__ void __launch_bounds__(LL_THREADS + 32, 1) loss_long_kernel(const __grid_constant__ Loss P)
{
    constexpr int E = BF16 ? 8 : 4, PER = LL_PIECE / 16 / LL_THREADS;                 // vectors of a piece to a thread
    using T = typename std::conditional<BF16, uint16_t, uint32_t>::type;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ __align__(8) unsigned long long bars[2 * LL_PIECES];
    __shared__ int s_index[LS_MAX_K], abort_flag;
    __shared__ float s_q[LS_MAX_K], s_loss[LL_WARPS];
    __shared__ Part s_part[LL_WARPS], s_teach[LL_WARPS];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int nvec = P.m / E, pieces = (nvec * 16 + LL_PIECE - 1) / LL_PIECE;
    auto full = [&](int s) { return smem_u32(&bars[s]); };
    auto empty = [&](int s) { return smem_u32(&bars[LL_PIECES + s]); };
    if (t == 0) {
        for (int s = 0; s < LL_PIECES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), LL_WARPS); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    int slot = 0;
    uint32_t ph = 0;
    auto advance = [&] { if (++slot == LL_PIECES) { slot = 0; ph ^= 1u; } };
    if (warp == LL_WARPS) {
        if (lane == 0) {
            bool ok = true;
            int issued = 0;
            for (long long row = blockIdx.x; row < P.rows && ok; row += gridDim.x) {
                const unsigned char *src = (const unsigned char *)((const T *)P.scores + (size_t)row * P.ld);
                for (int c = 0; c < pieces; ++c, advance()) {
                    if (!(ok = mbar_wait(empty(slot), ph ^ 1u, &abort_flag))) break;
                    const uint32_t bytes = (uint32_t)min(LL_PIECE, nvec * 16 - c * LL_PIECE);
                    mbar_expect_tx(full(slot), bytes);
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                                 ::"r"(smem_u32(ring) + slot * LL_PIECE), "l"(src + (size_t)c * LL_PIECE), "r"(bytes), "r"(full(slot)) : "memory");
                    if (issued < LL_PIECES) ++issued;
                }
            }
            // nothing may land in shared memory after the block has gone: the last copy into every piece, with a bound of its own
            int unused = 0, s = slot;
            for (int q = 0; q < issued; ++q) {
                if (--s < 0) { s = LL_PIECES - 1; ph ^= 1u; }
                mbar_wait(full(s), ph, &unused);
            }
        }
        return;
    }
    auto block_sync = [&] { asm volatile("bar.sync 1, %0;" ::"n"(LL_THREADS) : "memory"); };
    bool ok = true;
    const u64 c2 = pack2(P.c, P.c);
    for (long long row = blockIdx.x; row < P.rows; row += gridDim.x) {
        const float weight = P.weight ? P.weight[row] : 1.f;
        int named = -1;
        float logit = 0.f, score = 0.f;
        if (t < P.k) {
            named = P.index[(size_t)row * P.k + t];
            if (P.logits) logit = P.logits[(size_t)row * P.k + t];
        }
        // ---- maximum and sum
        const int slot0 = slot;
        const uint32_t ph0 = ph;
        Part part = {-INFINITY, 0.f};
        for (int c = 0; c < pieces; ++c, advance()) {
            ok = mbar_wait(full(slot), ph, &abort_flag) && ok;
            uint4 x[PER];
#pragma unroll
            for (int v = 0; v < PER; ++v) {
                const int j = v * LL_THREADS + t;
                x[v] = BF16 ? make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u) : make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u);
                if (c * (LL_PIECE / 16) + j < nvec) x[v] = *reinterpret_cast<const uint4 *>(ring + slot * LL_PIECE + j * 16);
            }
            float top = largest<BF16>(x[0]);
#pragma unroll
            for (int v = 1; v < PER; ++v) top = fmaxf(top, largest<BF16>(x[v]));
            if (top > part.m) {
                part.s *= ex2_fast((part.m - top) * P.c);                                // (of minus infinity: 0 times 0)
                part.m = top;
            }
            const u64 at2 = pack2(finite_max(part.m), finite_max(part.m));
            u64 sum[2] = {0ull, 0ull};
#pragma unroll
            for (int v = 0; v < PER; ++v)
#pragma unroll
                for (int i = 0; i < E / 2; ++i) sum[i & 1] = add2(sum[i & 1], exponentials(two<BF16>(x[v], i), at2, c2));
            float a, b;
            unpack2(add2(sum[0], sum[1]), a, b);
            part.s += a + b;
        }
        part = join<32>(part, P.c);
        // ---- the teacher
        Part teach = {-INFINITY, 0.f};
        if (named < 0 || named >= P.m) named = -1;
        const float l0 = named >= 0 ? logit : -INFINITY;
        if (warp * 32 < P.k) {
            teach.m = warp_max(l0);
            teach.s = ex2_fast((l0 - finite_max(teach.m)) * P.c);
#pragma unroll
            for (int off = 16; off; off /= 2) teach.s += __shfl_xor_sync(0xffffffffu, teach.s, off);
        }
        if (lane == 0) { s_part[warp] = part; s_teach[warp] = teach; }
        block_sync();
        if (named >= 0) {
            const int piece = slot0 + named / (LL_PIECE / (int)sizeof(T));
            const T *at = reinterpret_cast<const T *>(ring + (piece < LL_PIECES ? piece : piece - LL_PIECES) * LL_PIECE) + named % (LL_PIECE / (int)sizeof(T));
            score = BF16 ? __uint_as_float((uint32_t)*at << 16) : __uint_as_float((uint32_t)*at);
        }
        part = join<32>(lane < LL_WARPS ? s_part[lane] : Part{-INFINITY, 0.f}, P.c);
        part.s = __shfl_sync(0xffffffffu, part.s, 0);
        teach = join<32>(lane < LL_WARPS ? s_teach[lane] : Part{-INFINITY, 0.f}, P.c);
        teach.s = __shfl_sync(0xffffffffu, teach.s, 0);
        const bool live = teach.s != 0.f;                                             // (NaN, too)
        const float teach_at = finite_max(teach.m), teach_inv = live ? 1.f / teach.s : 0.f;
        float own_q = 0.f, sum = 0.f;
        if (warp * 32 < P.k) {
            const float log_all = logf(part.s) - logf(teach.s);
            own_q = ex2_fast((l0 - teach_at) * P.c) * teach_inv;
            if (own_q != 0.f) sum = own_q * (((l0 - teach_at) - (score - part.m)) * P.inv_t + log_all);
            if (t < P.k) { s_index[t] = named; s_q[t] = own_q; }
#pragma unroll
            for (int off = 16; off; off /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        }
        if (lane == 0) s_loss[warp] = ok ? sum : __uint_as_float(0x7fffffffu);
        // ---- the gradient
        const float w = weight * P.inv_t, a = w / part.s;
        T *out = (T *)P.grad + (size_t)row * P.ldg;
        const u64 at2 = pack2(part.m, part.m), f2 = pack2(a, a);
        slot = slot0;
        ph = ph0;
        for (int c = 0; c < pieces; ++c, advance()) {
            if (P.grad)
#pragma unroll
                for (int v = 0; v < PER; ++v) {
                    const int j = v * LL_THREADS + t, at = c * (LL_PIECE / 16) + j;
                    if (at >= nvec) break;
                    const uint4 x = *reinterpret_cast<const uint4 *>(ring + slot * LL_PIECE + j * 16);
                    uint32_t r[4];
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) {
                        float p, q;
                        unpack2(mul2(exponentials(two<BF16>(x, i), at2, c2), f2), p, q);
                        if constexpr (BF16) r[i] = bf16_pair(p, q);
                        else { r[2 * i] = __float_as_uint(p); r[2 * i + 1] = __float_as_uint(q); }
                    }
                    if (!live) r[0] = r[1] = r[2] = r[3] = 0u;
                    *reinterpret_cast<uint4 *>(out + (size_t)at * E) = make_uint4(r[0], r[1], r[2], r[3]);
                }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty(slot));
        }
        block_sync();
        if (t == 0) {
#pragma unroll
            for (int i = 1; i < LL_WARPS; ++i) sum += s_loss[i];
            P.loss[row] = live ? sum : 0.f;
        }
        // named entries: each by the first of those that name its column
        if (P.grad && live && named >= 0) {
            float q = 0.f;
            bool first = true;
            for (int o = 0; o < P.k; ++o)
                if (s_index[o] == named) {
                    first &= o >= t;
                    q += s_q[o];
                }
            if (first) {
                const float g = ex2_fast((score - part.m) * P.c) * a - q * w;
                out[named] = BF16 ? (T)bf16_pair(g, 0.f) : (T)__float_as_uint(g);
            }
        }
    }
}

template <bool BF16, int TPR, int V, int C, bool EVEN>
skb_status launch(const Loss &P, cudaStream_t st)
{
    constexpr int threads = TPR <= 256 ? 256 : TPR, groups = threads / TPR;
    const long long blocks = (P.rows + groups - 1) / groups * C;
    if (blocks > 0x7fffffffLL) return op_fail(SKB_ERR_SHAPE, "too many rows");
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = (size_t)groups * 4 * P.k * sizeof(float);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = C;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = C > 1 ? 1 : 0;
    cudaLaunchKernelEx(&cfg, loss_kernel<BF16, TPR, V, C, EVEN>, P);
    return op_launched("plan_loss");
}

template <bool BF16, bool EVEN>
skb_status launch_by_length(const Loss &P, long long vec, int sms, cudaStream_t st)
{
    // more blocks to a row than it needs where there are too few rows to fill the device
    const auto blocks = [&](int least) {
        int c = least;
        while (c < 8 && P.rows * c < 2 * sms && vec / (2 * c) >= 512) c *= 2;
        return c;
    };
    // Short rows are latency: several to a warp where there are more than the device's warps take at once, with more of a row to a thread where there are
    // many more.  (us in bf16, so / a warp to a row: 65536 rows of 64 12 / 36, of 256 15 / 39, of 512 25 / 42, of 1024 46 / 50; 4736 rows of 64 3.0 / 4.5; 2368
    // 2.9 / 3.4.  Eight vectors a thread for four: 65536 rows of 512 25 / 29, 9472 rows 5.8 / 5.4.  More than 32 entries would take too much shared memory.)
    if (P.k <= 32 && P.rows >= 16 * sms) {
        const bool many = P.rows >= 128 * sms;
        if (vec <= 8 * 4) return launch<BF16, 8, 4, 1, EVEN>(P, st);
        if (vec <= 8 * 8 && many) return launch<BF16, 8, 8, 1, EVEN>(P, st);
        if (vec <= 16 * 4) return launch<BF16, 16, 4, 1, EVEN>(P, st);
        if (vec <= 16 * 8 && many) return launch<BF16, 16, 8, 1, EVEN>(P, st);
    }
    // (us, rows of bf16 as the line says / as the next ones would: 256 vectors by a warp or by four, 1184 rows 10 / 10, 8192 20 / 28, 32768 51 / 89; 4096 vectors by a
    // block or by two and more, 148 rows 11 / 13, 592 21 / 26, 4096 92 / 110; 8192 vectors through shared memory or by a cluster, 100 rows 16 / 14, 148 rows
    // 16 / 19, 592 39 / 43, 4096 199 / 218; 12288 vectors, 1184 rows 92 / 113)
    if (vec <= 32 * 4) return launch<BF16, 32, 4, 1, EVEN>(P, st);
    if (vec <= 32 * 8 && P.rows >= 8 * sms) return launch<BF16, 32, 8, 1, EVEN>(P, st);
    if (vec <= 128 * 4) return launch<BF16, 128, 4, 1, EVEN>(P, st);
    if (vec > 256 * 8 && vec <= 512 * 8 && P.rows >= sms) return launch<BF16, 512, 8, 1, EVEN>(P, st);
    if (EVEN && vec > 512 * 8 && vec <= LL_PIECES * (LL_PIECE / 16) && P.rows >= sms) {
        constexpr int smem = LL_PIECES * LL_PIECE;
        cudaFuncSetAttribute(loss_long_kernel<BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        loss_long_kernel<BF16><<<sms, LL_THREADS + 32, smem, st>>>(P);
        return op_launched("plan_loss");
    }
    if (vec <= 256 * 8 * 8) {
        const int c = blocks(vec <= 256 * 8 ? 1 : vec <= 256 * 16 ? 2 : vec <= 256 * 32 ? 4 : 8);
        if (c == 1) return vec <= 256 * 4 ? launch<BF16, 256, 4, 1, EVEN>(P, st) : launch<BF16, 256, 8, 1, EVEN>(P, st);
        if (c == 2) return launch<BF16, 256, 8, 2, EVEN>(P, st);
        if (c == 4) return launch<BF16, 256, 8, 4, EVEN>(P, st);
        return launch<BF16, 256, 8, 8, EVEN>(P, st);
    }
    if (vec <= 512 * 8 * 8) return launch<BF16, 512, 8, 8, EVEN>(P, st);
    return launch<BF16, 512, 0, 8, EVEN>(P, st);
}
template <bool BF16>
skb_status launch_loss(const Loss &P, int sms, cudaStream_t st)
{
    constexpr int E = BF16 ? 8 : 4;
    // vectors that a row may touch: one more than it fills where rows do not all start on a 16-byte boundary
    const bool aligned = (uintptr_t)P.scores % 16 == 0 && P.ld % E == 0;
    const long long vec = ((long long)P.m + (aligned ? E - 1 : 2 * E - 2)) / E;
    const bool even = aligned && P.m % E == 0 && (!P.grad || ((uintptr_t)P.grad % 16 == 0 && P.ldg % E == 0));
    return even ? launch_by_length<BF16, true>(P, vec, sms, st) : launch_by_length<BF16, false>(P, vec, sms, st);
}

// Whether rows of the gradient and of the scores have entries in common, delta elements apart.  (Rows of different strides whose ranges meet: taken to.)
bool rows_overlap(long long delta, long long rows, long long m, long long ld, long long ldg)
{
    if (delta >= (rows - 1) * ld + m || -delta >= (rows - 1) * ldg + m) return false;
    if (rows == 1 || ld != ldg) return true;
    // gradient row j begins r after scores row j + q, and ld - r before the next
    const long long q = delta >= 0 ? delta / ld : -((-delta + ld - 1) / ld), r = delta - q * ld;
    const auto some = [&](long long apart) { return apart < rows && -apart < rows; };
    return (r < m && some(q)) || (ld - r < m && some(q + 1));
}

}  // namespace
}  // namespace skb

using namespace skb;

extern "C" skb_status sinkhorn_plan_loss(const void *scores, int dtype, long long rows, int m, long long ld, const int *index, const float *logits, int k,
                                         float temperature, const float *weight, float *loss, void *grad, long long ldg, void *stream)
{
    if (!scores || !index || !loss) return op_fail(SKB_ERR_NULL, "scores, index and loss are required");
    if (dtype != SKB_F32 && dtype != SKB_BF16) return op_fail(SKB_ERR_VALUE, "scores must be SKB_F32 or SKB_BF16");
    if (rows < 1 || rows > 0x7fffffffLL || m < 1 || m > 262143 || k < 1 || k > LS_MAX_K)
        return op_fail(SKB_ERR_SHAPE, "rows from 1 to 2^31 - 1, m from 1 to 262143 and k from 1 to 256 are supported");
    if (ld < m || (grad && ldg < m)) return op_fail(SKB_ERR_SHAPE, "rows must not overlap: ld and ldg at least m");
    if (!(temperature >= 1e-30f && temperature <= 1e30f)) return op_fail(SKB_ERR_VALUE, "temperature must be from 1e-30 to 1e30");
    const uintptr_t size = dtype == SKB_BF16 ? 2 : 4;
    if ((uintptr_t)scores % size || (uintptr_t)grad % size || (uintptr_t)index % 4 || (uintptr_t)logits % 4 || (uintptr_t)weight % 4 || (uintptr_t)loss % 4)
        return op_fail(SKB_ERR_WORKSPACE, "arrays must be aligned to their types");
    if (grad == scores && ldg != ld) return op_fail(SKB_ERR_SHAPE, "a gradient in the place of the scores has their row stride");
    if (grad && grad != scores && rows_overlap(((long long)(uintptr_t)grad - (long long)(uintptr_t)scores) / (long long)size, rows, m, ld, ldg))
        return op_fail(SKB_ERR_VALUE, "a gradient that overlaps the scores must be in their place");
    int dev = 0, sms = 0;
    cudaGetDevice(&dev);
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return op_launched("device");
    const Loss P = {scores, index, logits, weight, loss, grad, rows, ld, ldg, m, k, 1.f / temperature, (float)(1.4426950408889634 / (double)temperature)};
    return dtype == SKB_BF16 ? launch_loss<true>(P, sms, (cudaStream_t)stream) : launch_loss<false>(P, sms, (cudaStream_t)stream);
}
