// One row of a coupling held as weights w_j in [0, 1] (the largest is 1): the cuts by top-k, top-p and min-p, and draws.
//
// The order of a row's entries is w descending, equal ones by their index.  A cut is a weight and an index: kept are the
// entries with w > tau, and those with w = tau up to index J.  It is found by bisection of the weight's bit pattern (an
// integer that grows with the weight): every pass adds up the entries above a pivot, until at most 32 lie between
// the pivots, which are sorted.  Draws look for the first entry whose cumulative kept weight, in the order of the indices,
// exceeds u times the total: by sums of 128 entries, then inside one of them.
//
// `Real` is float where the weights are fp32.  Every comparison that decides something is then checked against bounds on
// the errors (RowError), and a row with a comparison inside them is `unsure`: its caller decides it again with better
// weights, in the end with exact ones, which takes what it finds.  Sums are in double and always added in one order: results do not depend on timing.
#pragma once
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

namespace skb {

constexpr int ROW_TILE = 128;          // entries of a partial sum; rows are padded to whole tiles with weights of zero
constexpr int ROW_CAND = 32;

// What a group of whole warps shares: scratch in shared memory.
struct RowScratch {
    double mass[16];
    int count[16];
    union {
        struct {
            double cand_w[ROW_CAND], sort_w[ROW_CAND];
            int cand_j[ROW_CAND], sort_j[ROW_CAND];
        };
        unsigned part[2][16][6];       // (skb_draw_quick.cuh)
    };
    int n_cand, tie_j, band[3];
};
struct RowGroup {
    int t, nt, bar;                    // thread in the group, threads, named barrier
    RowScratch *sc;
    __device__ __forceinline__ void sync() const
    {
        if (nt == 32) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(nt) : "memory");
    }
    // sums over the group, the same in every thread
    __device__ __noinline__ void add(double &mass, int &count) const
    {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            mass += __shfl_xor_sync(0xffffffffu, mass, off);
            count += __shfl_xor_sync(0xffffffffu, count, off);
        }
        if (nt == 32) return;
        if ((t & 31) == 0) { sc->mass[t >> 5] = mass; sc->count[t >> 5] = count; }
        sync();
        mass = 0.0; count = 0;
#pragma unroll 1
        for (int i = 0; i < nt >> 5; ++i) { mass += sc->mass[i]; count += sc->count[i]; }
        sync();
    }
    template <typename Real>
    __device__ __forceinline__ Real largest(Real v) const
    {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, off));
        if (nt == 32) return v;
        if ((t & 31) == 0) sc->mass[t >> 5] = (double)v;
        sync();
#pragma unroll 1
        for (int i = 0; i < nt >> 5; ++i) v = fmax(v, (Real)sc->mass[i]);
        sync();
        return v;
    }
};

__device__ __forceinline__ int weight_bits(float v) { return __float_as_int(v); }
__device__ __forceinline__ long long weight_bits(double v) { return __double_as_longlong(v); }
__device__ __forceinline__ float weight_of(int b) { return __int_as_float(b); }
__device__ __forceinline__ double weight_of(long long b) { return __longlong_as_double(b); }
__device__ __forceinline__ void load4(const float *p, float (&v)[4])
{
    const float4 a = *reinterpret_cast<const float4 *>(p);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
__device__ __forceinline__ void load4(const double *p, double (&v)[4])
{
    const double2 a = reinterpret_cast<const double2 *>(p)[0], b = reinterpret_cast<const double2 *>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}

// Settings of a lane, already checked: k entries (INT_MAX: all), share p of the mass (>= 1: all), smallest weight r.
struct RowCuts {
    int k;
    double p;
    float r;
};

// Bounds on what is compared: two sums of a row's weights are off by `sums` between them, two weights at 2^-q of the
// largest by `weight + slope q` of themselves.  All zero: exact.
struct RowError {
    double sums;
    float weight, slope;
    __device__ __forceinline__ bool any() const { return sums != 0.0; }     // (a bound that is NaN: nothing is sure)
};

template <typename Real>
struct RowCut {
    Real tau;
    int J;
    double mass;                       // of what is kept, and its number
    int count;
    Real lowest;                       // smallest weight that a cut was made at; 1 where there was none
    __device__ __forceinline__ bool kept(Real w, int j) const { return w > tau || (w == tau && j <= J); }
};

// Shrinks the cut to the shortest head of the order that has `target` entries, or, by mass, a mass of `target`; the
// present cut has more.
template <typename Real>
__device__ __noinline__ void row_find(const Real *w, const int mp, const RowGroup &G, const bool by_mass, const double target, RowCut<Real> &cut,
                         const RowError &err, bool &unsure)
{
    const RowCut<Real> old = cut;
    Real lo = old.tau > 0 ? old.tau : weight_of((decltype(weight_bits(Real(0))))1), hi = Real(2);
    int n_lo = old.count, n_hi = 0;
    double m_hi = 0.0;
    bool first = true;
#pragma unroll 1
    while (n_lo - n_hi > ROW_CAND) {
        const auto bl = weight_bits(lo), bh = weight_bits(hi);
        if (bh - bl <= 1) break;                                    // equal weights
        auto bp = bl + (bh - bl) / 2;
        // what is below (mass - target) / count adds up to less than mass - target: the border is above it
        // (and few cuts by rank need what is below 2^-30)
        if (first) bp = weight_bits((Real)(by_mass ? (old.mass - target) / n_lo : 9.3e-10));
        first = false;
        if (bp <= bl) bp = bl + 1;
        if (bp >= bh) bp = bh - 1;
        const Real pivot = weight_of(bp);
        double s4[4] = {0, 0, 0, 0};
        int c = 0;
#pragma unroll 1
        for (int j = 4 * G.t; j < mp; j += 4 * G.nt) {
            Real v[4];
            load4(w + j, v);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v[i] >= pivot) { s4[i] += (double)v[i]; ++c; }
        }
        double s = (s4[0] + s4[1]) + (s4[2] + s4[3]);
        G.add(s, c);
        if ((by_mass ? s : (double)c) >= target) { lo = pivot; n_lo = c; }
        else { hi = pivot; n_hi = c; m_hi = s; }
    }
    const int have = n_lo - n_hi, lane = G.t & 31;
    if (have > ROW_CAND) {
        // more than a warp of entries that all weigh lo: the first so many of them by index
        if (err.any()) { unsure = true; return; }
        double need = by_mass ? ceil((target - m_hi) / (double)lo) : target - n_hi;
        need = fmin(fmax(need, 1.0), (double)have);
        const int r = (int)need;
        if (G.t < 32) {
            int seen = 0, at = -1;
#pragma unroll 1
            for (int j = lane; j < mp && at < 0; j += 32) {
                const bool is = w[j] == lo && (lo != old.tau || j <= old.J);
                const unsigned ball = __ballot_sync(0xffffffffu, is);
                if (seen + __popc(ball) >= r) {
                    unsigned left = ball;
#pragma unroll 1
                    for (int q = r - seen; q > 1; --q) left &= left - 1;
                    at = j - lane + __ffs(left) - 1;
                }
                seen += __popc(ball);
            }
            if (lane == 0) G.sc->tie_j = at;
        }
        G.sync();
        cut.tau = lo; cut.J = G.sc->tie_j; cut.mass = m_hi + need * (double)lo; cut.count = n_hi + r;
        G.sync();
        return;
    }
    if (G.t == 0) G.sc->n_cand = 0;
    G.sync();
#pragma unroll 1
    for (int j = 4 * G.t; j < mp; j += 4 * G.nt) {
        Real v[4];
        load4(w + j, v);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (v[i] >= lo && v[i] < hi && (v[i] != old.tau || j + i <= old.J)) {
                const int q = atomicAdd(&G.sc->n_cand, 1);
                if (q < ROW_CAND) { G.sc->cand_w[q] = (double)v[i]; G.sc->cand_j[q] = j + i; }
            }
    }
    G.sync();
    const int n = min(G.sc->n_cand, ROW_CAND);
    if (G.t < 32 && lane < n) {
        const double mine = G.sc->cand_w[lane];
        const int j = G.sc->cand_j[lane];
        int rank = 0;
#pragma unroll 1
        for (int q = 0; q < n; ++q) {
            const double o = G.sc->cand_w[q];
            rank += o > mine || (o == mine && G.sc->cand_j[q] < j) ? 1 : 0;
        }
        G.sc->sort_w[rank] = mine;
        G.sc->sort_j[rank] = j;
    }
    G.sync();
    const double mine = lane < n ? G.sc->sort_w[lane] : 0.0;
    const int j = lane < n ? G.sc->sort_j[lane] : -1;
    G.sync();
    double sum = mine;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
        const double o = __shfl_up_sync(0xffffffffu, sum, off);
        if (lane >= off) sum += o;
    }
    const unsigned reach = __ballot_sync(0xffffffffu, lane < n && (by_mass ? m_hi + sum : (double)(n_hi + lane + 1)) >= target);
    const int at = reach ? __ffs(reach) - 1 : n - 1;
    const double w_at = __shfl_sync(0xffffffffu, mine, at), m_at = m_hi + __shfl_sync(0xffffffffu, sum, at);
    if (by_mass && err.any() && !(m_at - target > err.sums && target - (m_at - w_at) > err.sums)) unsure = true;
    cut.tau = (Real)w_at;
    cut.J = __shfl_sync(0xffffffffu, j, at);
    cut.mass = m_at;
    cut.count = n_hi + at + 1;
}

// Cuts a row and leaves the sums of its tiles' kept weights in `tiles`.  `count` entries are above zero and have the mass
// `mass`, `top` is the largest (1 up to errors).  Returns false where the row is unsure.
template <typename Real>
__device__ __noinline__ bool row_cut(const Real *w, const int mp, const RowGroup &G, const RowCuts &want, const Real top, const double mass, const int count,
                        const RowError &err, RowCut<Real> &cut, double *tiles)
{
    bool unsure = false;
    cut.tau = 0; cut.J = -1; cut.mass = mass; cut.count = count; cut.lowest = 1;
    Real border[3] = {0, 0, 0};                 // of each cut that was made
    if (want.k < cut.count) {
        row_find(w, mp, G, false, (double)want.k, cut, err, unsure);
        border[0] = cut.tau;
    }
    if (unsure) return false;
    if (want.p < 1.0) {
        row_find(w, mp, G, true, want.p * cut.mass, cut, err, unsure);
        border[1] = cut.tau;
    }
    if (unsure) return false;
    if (want.r > 0.f) {
        border[2] = (Real)want.r * top;
        if (border[2] > cut.tau) { cut.tau = border[2]; cut.J = 0x7fffffff; }
    }
#pragma unroll
    for (int q = 0; q < 3; ++q)
        if (border[q] > 0 && border[q] < cut.lowest) cut.lowest = border[q];
    const bool look = err.any() && (border[0] > 0 || border[1] > 0 || border[2] > 0);
    Real low[3], high[3];
    int near_[3] = {0, 0, 0};
    if (look) {
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            const double e = border[q] > 0 ? (double)(err.weight - err.slope * fminf(log2f((float)border[q]), 0.f)) : 0.0;
            low[q] = (Real)(border[q] * (1.0 - e));
            high[q] = border[q] > 0 ? (Real)(border[q] * (1.0 + e)) : Real(-1);
        }
        if (G.t < 3) G.sc->band[G.t] = 0;
        G.sync();
    }
    const int lane = G.t & 31;
#pragma unroll 1
    for (int q = G.t >> 5; q < mp / ROW_TILE; q += G.nt >> 5) {
        const int j = q * ROW_TILE + 4 * lane;
        Real v[4];
        double s = 0.0;
        load4(w + j, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (cut.kept(v[i], j + i)) s += (double)v[i];
            if (look) {
#pragma unroll
                for (int b = 0; b < 3; ++b) near_[b] += v[i] >= low[b] && v[i] <= high[b] ? 1 : 0;
            }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        if (lane == 0) tiles[q] = s;
    }
    if (look) {
#pragma unroll
        for (int b = 0; b < 3; ++b) {
            const int c = __reduce_add_sync(0xffffffffu, near_[b]);
            if (lane == 0 && c) atomicAdd(&G.sc->band[b], c);
        }
    }
    G.sync();
    if (look) {
        // the entry at the border of a rank or a mass, and no other; none at that of a size
        const bool clear = (border[0] > 0 ? G.sc->band[0] <= 1 : true) && (border[1] > 0 ? G.sc->band[1] <= 1 : true) &&
                           (border[2] > 0 ? G.sc->band[2] == 0 : true);
        G.sync();
        if (!clear) return false;
    }
    return true;
}

// Total of the tiles' sums; by one warp.
__device__ __forceinline__ double row_total(const double *tiles, const int ntiles)
{
    double s = 0.0;
#pragma unroll 1
    for (int q = threadIdx.x & 31; q < ntiles; q += 32) s += tiles[q];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    return s;
}

// One draw, by one warp: the entry's index and weight.  Returns false where it is unsure.
template <typename Real>
__device__ __noinline__ bool row_draw(const Real *w, const RowCut<Real> &cut, const double *tiles, const int ntiles, const double total, const double u,
                         const RowError &err, int &index, double &weight)
{
    const int lane = threadIdx.x & 31;
    const double target = u * total;
    // the first tile whose cumulative sum is above the target, or the last one that has something
    double base = 0.0, before = 0.0;
    int tile = -1;
#pragma unroll 1
    for (int q0 = 0; q0 < ntiles; q0 += 32) {
        const double v = q0 + lane < ntiles ? tiles[q0 + lane] : 0.0;
        double s = v;
#pragma unroll
        for (int off = 1; off < 32; off *= 2) {
            const double o = __shfl_up_sync(0xffffffffu, s, off);
            if (lane >= off) s += o;
        }
        const unsigned some = __ballot_sync(0xffffffffu, v > 0.0), over = __ballot_sync(0xffffffffu, v > 0.0 && base + s > target);
        if (over || some) {
            const int at = over ? __ffs(over) - 1 : 31 - __clz((int)some);
            tile = q0 + at;
            before = base + __shfl_sync(0xffffffffu, s - v, at);
        }
        base += __shfl_sync(0xffffffffu, s, 31);
        if (over) break;
    }
    index = -1;
    weight = 0.0;
    if (tile < 0) return false;                      // no weight at all, or none that is a number
    const int j = tile * ROW_TILE + 4 * lane;
    Real v[4];
    load4(w + j, v);
    double own = 0.0;
    bool kept[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { kept[i] = v[i] > 0 && cut.kept(v[i], j + i); own += kept[i] ? (double)v[i] : 0.0; }
    double s = own;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
        const double o = __shfl_up_sync(0xffffffffu, s, off);
        if (lane >= off) s += o;
    }
    double run = before + (s - own), at_w = 0.0, at_run = 0.0, last_w = 0.0, last_run = 0.0;
    int at_j = -1, last_j = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (kept[i]) {
            run += (double)v[i];
            if (at_j < 0 && run > target) { at_j = j + i; at_w = (double)v[i]; at_run = run; }
            last_j = j + i; last_w = (double)v[i]; last_run = run;
        }
    const unsigned over = __ballot_sync(0xffffffffu, at_j >= 0), some = __ballot_sync(0xffffffffu, last_j >= 0);
    if (!over && lane == 31 - __clz((int)some)) { at_j = last_j; at_w = last_w; at_run = last_run; }
    const int who = over ? __ffs(over) - 1 : 31 - __clz((int)some);
    index = __shfl_sync(0xffffffffu, at_j, who);
    weight = __shfl_sync(0xffffffffu, at_w, who);
    const double end = __shfl_sync(0xffffffffu, at_run, who);
    return !err.any() || (end - target > err.sums && target - (end - weight) > err.sums);
}

}  // namespace skb
