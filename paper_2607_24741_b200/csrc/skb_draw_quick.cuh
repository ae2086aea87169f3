// One row of fp32 weights cut and drawn from in a hurry: bounds on all errors known, sums as integers, no sorting.
//
// Sums are counted in units of 2^-30 of the row's mass: a thread adds its weights in fp32, rounds the sum to units, and the
// warp's are added by one integer reduction, exactly and in no particular order.  A cut is found by three pivots at a time,
// quarters of the bracket's bit patterns.  As soon as a quarter of the row is left, the weights in the bracket move to a
// list, which later passes read (a pass is nine instructions a weight); when 32 are left, each counts and adds up those
// above it, which ends the search.  Two weights within their errors of each other leave the row unsure, so no ties have to be
// ordered here.  skb_draw_row.cuh has the careful form.
//
// Error of a comparison: a sum over a part of the row against a share f of its mass M, sum - f M = (1 - f) part - f rest.  Where
// part is about f M, relative errors of the weights of at most e move that by 2 f (1 - f) e M, and no more.
#pragma once
#include "skb_draw_row.cuh"

namespace skb {

constexpr float QUICK_ONE = 1073741824.f;                        // units of a row's mass

// Sums over the group of N counts each thread has; the same in all threads.  `turn` alternates between two buffers, so that
// one barrier does.
template <int N>
__device__ __forceinline__ void group_add(const RowGroup &G, unsigned (&v)[N], int &turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __reduce_add_sync(0xffffffffu, v[i]);
    if (G.nt == 32) return;
    turn ^= 1;
    if ((G.t & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) G.sc->part[turn][G.t >> 5][i] = v[i];
    G.sync();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        unsigned s = 0;
#pragma unroll 1
        for (int q = 0; q < G.nt >> 5; ++q) s += G.sc->part[turn][q][i];
        v[i] = s;
    }
}
// What a sum and a share f of the row's mass may be apart, in units: errors of the weights, of additions and of rounding to units.
struct QuickSlack {
    float weights, rest;                // (and 130 units, of a target's own rounding)
    __device__ __forceinline__ unsigned at(float f) const { return (unsigned)(2.f * f * (1.f - f) * weights + rest) + 130u; }
};

struct QuickCut {
    float tau;                          // kept: weights from here on
    unsigned count, mass;               // of what is kept; mass in units
    unsigned own;                       // this thread's of `count`
};

// Quadruples of a row that a thread has: whole tiles to a warp, one after the other.
struct Span {
    int begin, end, step;
    __device__ __forceinline__ Span(const RowGroup &G, int mp)
    {
        const int nw = G.nt >> 5, gw = G.t >> 5, tiles = mp / ROW_TILE;
        begin = tiles * gw / nw * ROW_TILE + 4 * (G.t & 31);
        end = tiles * (gw + 1) / nw * ROW_TILE;
        step = ROW_TILE;
    }
};

// Exclusive sum over the group's threads of a count each.
__device__ __forceinline__ unsigned group_offset(const RowGroup &G, const unsigned v, int &turn)
{
    const int lane = G.t & 31;
    unsigned s = v;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
        const unsigned o = __shfl_up_sync(0xffffffffu, s, off);
        if (lane >= off) s += o;
    }
    unsigned before = s - v;
    if (G.nt == 32) return before;
    turn ^= 1;
    if (lane == 31) G.sc->part[turn][G.t >> 5][0] = s;
    G.sync();
#pragma unroll 1
    for (int q = 0; q < G.t >> 5; ++q) before += G.sc->part[turn][q][0];
    return before;
}

// Where a search has come to: the border is in [lo, hi), n weights and m units are from there on.
struct QuickBracket {
    int lo, hi;
    unsigned n_lo, m_lo, n_hi, m_hi;
};

// The border among the n <= QUICK_FEW weights w (zeros up to a whole quadruple), n_out weights and m_out units being above all
// of them: every thread counts and adds up what is above its weight.  By each warp of the group for itself.  Leaves the
// bracket's sums around the border, its weight, and the weights next to it in `below` and `above`.
constexpr int QUICK_FEW = 32;
__device__ __forceinline__ bool quick_rank(const float *w, const int n, const bool by_mass, const unsigned target, const float unit, const unsigned n_out,
                                           const unsigned m_out, QuickBracket &B, unsigned &at, unsigned &below, unsigned &above)
{
    const int lane = threadIdx.x & 31;
    const float x = lane < n ? w[lane] : 0.f;
    float s = 0.f;
    unsigned c = 0;
#pragma unroll 2
    for (int j = 0; j < n; j += 4) {
        float v[4];
        load4(w + j, v);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (v[i] > x) { ++c; s += v[i]; }
    }
    const unsigned b = __float_as_uint(x), m0 = m_out + __float2uint_rn(s * unit), m1 = m_out + __float2uint_rn((s + x) * unit);
    const bool is = (int)b >= B.lo && (int)b < B.hi && (by_mass ? m0 < target && m1 >= target : n_out + c + 1 == target);
    const unsigned ball = __ballot_sync(0xffffffffu, is);
    if (!ball) return false;                                     // two that are equal, or a sum that was rounded past the target
    const int who = __ffs(ball) - 1;
    at = __shfl_sync(0xffffffffu, b, who);
    B.n_lo = n_out + __shfl_sync(0xffffffffu, c, who) + 1;
    B.m_lo = __shfl_sync(0xffffffffu, m1, who);
    B.m_hi = __shfl_sync(0xffffffffu, m0, who);
    below = max(below, __reduce_max_sync(0xffffffffu, b < at ? b : 0u));
    above = min(above, __reduce_min_sync(0xffffffffu, b > at ? b : 0xffffffffu));
    return __popc(__ballot_sync(0xffffffffu, b == at)) == 1;
}

// Shrinks the cut to the shortest head with `target` entries, or units of mass.  `list` has room for `room` weights and
// QUICK_FEW more.  Returns false where it is unsure.
__device__ __forceinline__ bool quick_find(const float *row, const int mp, const RowGroup &G, const bool by_mass, const unsigned target, const float unit,
                                           const unsigned slack, const RowError &err, float *list, const unsigned room, QuickCut &cut, int &turn)
{
    QuickBracket B = {cut.tau > 0.f ? __float_as_int(cut.tau) : 1, __float_as_int(2.f), cut.count, cut.mass, 0u, 0u};
    unsigned own_lo = cut.own, own_hi = 0;
    const float *w = row;
    const Span all(G, mp);
    Span span = all;
    int n = mp;
    unsigned n_out = 0, m_out = 0;                               // number and mass of what is above all that w holds
    unsigned at = 0, below = 0, above = (unsigned)B.hi;          // the border, and what is next to it (beyond a list: its bracket)
    bool first = true;
#pragma unroll 1
    while (true) {
        const unsigned left = B.n_lo - B.n_hi;
        if (n > QUICK_FEW && (left <= QUICK_FEW || (w == row && left <= room))) {
            // what is in the bracket to a list, zeros behind it up to whole quadruples
            float *to = left <= QUICK_FEW ? list + room : list;
            unsigned next = group_offset(G, own_lo - own_hi, turn);
#pragma unroll 1
            for (int j = span.begin; j < span.end; j += span.step) {
                float x[4];
                load4(w + j, x);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (__float_as_int(x[i]) >= B.lo && __float_as_int(x[i]) < B.hi) to[next++] = x[i];
            }
            n = (int)((left + 3) / 4 * 4);
            if (G.t < n - (int)left) to[left + G.t] = 0.f;
            G.sync();
            w = to; below = (unsigned)B.lo - 1u; above = (unsigned)B.hi; n_out = B.n_hi; m_out = B.m_hi;
            span.begin = 4 * G.t; span.end = n; span.step = 4 * G.nt;
            own_lo = own_hi = 0;
            if (n > QUICK_FEW)
#pragma unroll 1
                for (int j = span.begin; j < span.end; j += span.step) own_lo += (unsigned)min(4, (int)left - j);
        }
        if (n <= QUICK_FEW) {
            if (!quick_rank(w, n, by_mass, target, unit, n_out, m_out, B, at, below, above)) return false;
            break;
        }
        const int gap = B.hi - B.lo;
        if (gap < 16) return false;                              // equal weights, or nearly
        int p[3] = {B.lo + gap / 4, B.lo + gap / 2, B.lo + gap / 4 * 3};
        if (first) {
            // below (mass - target) / count there is less than mass - target: the border is above; and few rows need
            // more than 2^-24 of their largest weight
            const int b = by_mass ? __float_as_int((float)(B.m_lo - target) / ((float)B.n_lo * unit) * 0.999f) : __float_as_int(5.9604645e-8f);
            if (b > B.lo && b < __float_as_int(0.25f)) {
                const int gap1 = __float_as_int(1.f) - b;
                p[0] = b; p[1] = b + gap1 / 3; p[2] = b + gap1 / 3 * 2;
            }
            first = false;
        }
        const float pv[3] = {__int_as_float(p[0]), __int_as_float(p[1]), __int_as_float(p[2])};
        float s[3] = {0.f, 0.f, 0.f};
        unsigned v[6] = {0, 0, 0, 0, 0, 0};
#pragma unroll 2
        for (int j = span.begin; j < span.end; j += span.step) {
            float x[4];
            load4(w + j, x);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int q = 0; q < 3; ++q)
                    if (x[i] >= pv[q]) { s[q] += x[i]; ++v[q]; }
        }
        const unsigned own[3] = {v[0], v[1], v[2]};
#pragma unroll
        for (int q = 0; q < 3; ++q) v[3 + q] = __float2uint_rn(s[q] * unit);
        group_add(G, v, turn);
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            const unsigned c = n_out + v[q], m = m_out + v[3 + q];
            if ((by_mass ? m : c) >= target) { if (p[q] > B.lo) { B.lo = p[q]; B.n_lo = c; B.m_lo = m; own_lo = own[q]; } }
            else if (p[q] < B.hi) { B.hi = p[q]; B.n_hi = c; B.m_hi = m; own_hi = own[q]; }
        }
    }
    cut.tau = __uint_as_float(at);
    cut.count = B.n_lo;
    cut.mass = B.m_lo;
    cut.own = 0;
    G.sync();                                                    // the list is read
    if (by_mass && !(B.m_lo > target + slack && target > B.m_hi + slack)) return false;
    const float e = err.weight - err.slope * fminf(log2f(cut.tau), 0.f);
    return cut.tau - __uint_as_float(below) > e * cut.tau && __uint_as_float(above) - cut.tau > e * cut.tau;
}

// Cuts the row.
__device__ __forceinline__ bool quick_cut(const float *w, const int mp, const RowGroup &G, const int k, const float p, const float smallest, const unsigned count, const unsigned own,
                                          const float unit, const QuickSlack &slack, const float sums, const RowError &err, float *list, const unsigned room, QuickCut &cut, int &turn)
{
    cut = {0.f, count, (unsigned)QUICK_ONE, own};
    // by rank, then by mass (one body: the code has to stay in the instruction cache)
#pragma unroll 1
    for (int by_mass = 0; by_mass < 2; ++by_mass) {
        if (by_mass ? p >= 1.f || cut.count <= 1 : (unsigned)k >= count) continue;
        if (by_mass && cut.tau > 0.f) {
            const Span all(G, mp);
#pragma unroll 1
            for (int j = all.begin; j < all.end; j += all.step) {
                float x[4];
                load4(w + j, x);
#pragma unroll
                for (int i = 0; i < 4; ++i) cut.own += x[i] >= cut.tau;
            }
        }
        // (a target by mass is off by 64 units: fp32's last place)
        const unsigned target = by_mass ? (unsigned)(p * (float)cut.mass) : (unsigned)k;
        if (!quick_find(w, mp, G, by_mass != 0, target, unit, slack.at(p) + (unsigned)sums, err, list, room, cut, turn)) return false;
    }
    if (smallest > 0.f) {
        const float e = err.weight - err.slope * log2f(smallest);
        const float low = smallest * (1.f - e), high = smallest * (1.f + e);
        unsigned near_[1] = {0};
        const Span all(G, mp);
#pragma unroll 2
        for (int j = all.begin; j < all.end; j += all.step) {
            float x[4];
            load4(w + j, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) near_[0] += x[i] >= low && x[i] <= high;
        }
        // (a smallest share of 1 keeps the largest weight, which is 1 itself)
        group_add(G, near_, turn);
        if (near_[0] != (smallest == 1.f ? 1u : 0u)) return false;
        cut.tau = fmaxf(cut.tau, smallest);
    }
    return true;
}

__device__ __forceinline__ bool quick_kept(float v, float tau) { return tau > 0.f ? v >= tau : v > 0.f; }

// Units of the kept weights by tile.
__device__ __forceinline__ void quick_tiles(const float *w, const int ntiles, const RowGroup &G, const float tau, const float unit, unsigned *tiles)
{
    const int lane = G.t & 31;
#pragma unroll 2
    for (int q = G.t >> 5; q < ntiles; q += G.nt >> 5) {
        float v[4], s = 0.f;
        load4(w + q * ROW_TILE + 4 * lane, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) s += quick_kept(v[i], tau) ? v[i] : 0.f;
        const unsigned u = __reduce_add_sync(0xffffffffu, __float2uint_rn(s * unit));
        if (lane == 0) tiles[q] = u;
    }
}
__device__ __forceinline__ unsigned quick_total(const unsigned *tiles, const int ntiles)
{
    unsigned s = 0;
#pragma unroll 1
    for (int q = threadIdx.x & 31; q < ntiles; q += 32) s += tiles[q];
    return __reduce_add_sync(0xffffffffu, s);
}
__device__ __forceinline__ unsigned warp_scan(unsigned v)          // inclusive
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
        const unsigned o = __shfl_up_sync(0xffffffffu, v, off);
        if (lane >= off) v += o;
    }
    return v;
}
// One draw, by one warp; false where it is unsure.
__device__ __forceinline__ bool quick_draw(const float *w, const int ntiles, const float tau, const float unit, const unsigned *tiles, const unsigned total,
                                           const float u, const QuickSlack &of, int &index, float &weight)
{
    const int lane = threadIdx.x & 31;
    // (u in units of 2^-32: what that cuts off moves the target by less than a unit)
    const unsigned target = __umulhi((unsigned)(u * 4294967296.f), total), slack = of.at(u);
    unsigned before = 0;
    int tile = -1;
#pragma unroll 1
    for (int q0 = 0; q0 < ntiles; q0 += 32) {
        const unsigned v = q0 + lane < ntiles ? tiles[q0 + lane] : 0u, s = before + warp_scan(v);
        const unsigned over = __ballot_sync(0xffffffffu, s > target);
        if (over) {
            const int at = __ffs(over) - 1;
            tile = q0 + at;
            before = __shfl_sync(0xffffffffu, s - v, at);
            break;
        }
        before = __shfl_sync(0xffffffffu, s, 31);
    }
    if (tile < 0) return false;
    float v[4], s = 0.f;
    load4(w + tile * ROW_TILE + 4 * lane, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = quick_kept(v[i], tau) ? v[i] : 0.f; s += v[i]; }
    const unsigned own = __float2uint_rn(s * unit), run = before + warp_scan(own);
    const unsigned over = __ballot_sync(0xffffffffu, run > target);
    if (!over) return false;
    const int who = __ffs(over) - 1;
    // among the thread's four: the first at which the sum passes the target
    const unsigned base = run - own;
    float sum = 0.f, wi = 0.f;
    int j = -1;
    unsigned start = 0, end = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned a = base + __float2uint_rn(sum * unit);
        sum += v[i];
        const unsigned b = base + __float2uint_rn(sum * unit);
        if (j < 0 && b > target) { j = tile * ROW_TILE + 4 * lane + i; wi = v[i]; start = a; end = b; }
    }
    const bool clear = j >= 0 && end > target + slack && target > start + slack;
    index = __shfl_sync(0xffffffffu, j, who);
    weight = __shfl_sync(0xffffffffu, wi, who);
    return __shfl_sync(0xffffffffu, (int)clear, who) != 0;
}

}  // namespace skb
