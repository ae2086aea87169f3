// Partners drawn from the rows of a coupling: row i of a lane is the distribution over j with weights
//     w_j = 2^(z_j - max z),  z_j = k (g_j - |x_i - y_j|^2),  k = log2(e) / (eps T),
// cut down by top-k, top-p and min-p (skb_draw_row.cuh), and a draw for each uniform number that is given.  The row's own
// potential drops out.  The plan is not stored: a warp (long rows: four, or a block) forms the weights of a row in shared
// memory, cuts and draws, and goes on to its next row.
//
// The indices are those of the definition in float64.  The weights are formed in fp32, with bounds on their errors, cut and drawn
// from (skb_draw_quick.cuh).  A row in which some comparison falls inside the bounds is formed again, to fp32's last place,
// where it weighs more than 2^-22 of its largest entry, and decided again with sums in double (skb_draw_row.cuh); what that
// leaves open goes on a list, for a kernel that decides in float64 throughout.
//
// Two ways to the exponents:
//   differences   |x - y|^2 in fp32 from a transposed copy of y: two operations a dimension and pair, two columns to an
//                 instruction; several rows at a time where that pays, so that a column's coordinates serve them all
//   products      deep bf16 and 4-bit clouds: x . y from the tensor cores (skb_dots.cu), 512 MB at a time,
//                 z = k (g - |y|^2) + 2 k x . y
// Rows that do not fit shared memory (from some 23 000 entries on), and rows whose exponents are too large for fp32 to hold a
// weight to a per cent, are decided in float64 alone, weights in the workspace.
//
// What bounds it: instructions of the searches and draws, not the exponentials.  256 lanes of 512 x 512, d = 15, top-p (131072
// rows, 67 M pairs): 0.70 ms, some 2900 instructions of a warp a row, of which forming and exponentials are a fifth (15 us at
// the rate of the exponentials); issue slots are used to 54 % and neither 16 nor 32 warps an SM instead of 24 change the time.
// 2 lanes of 8192 x 8192, d = 3, top-k 16, four draws: 0.77 ms, a list of some 50 entries a row, latencies of one warp's search between
// the block's barriers, 0.15 of it log probabilities of large exponents.  64 lanes of 1024 x 1024, d = 512 (bf16), top-p: 0.75 ms, of which products 0.18, rows 0.28, rows
// formed again 0.19 (2.7 % of them), norms 0.04, float64 0.09 (some ten rows, a cold kernel's latency).  Deep fp32 clouds, without tensor cores: 64 lanes of
// 1024 x 1024, d = 512, 25 ms.
#include <cuda_runtime.h>
#include <math_constants.h>
#include <algorithm>
#include <limits.h>

#include "skb_cloud4.cuh"
#include "skb_draw_quick.cuh"
#include "skb_draw_row.cuh"
#include "skb_f32x2.cuh"
#include "skb_operators.h"

namespace skb {
namespace {

constexpr int DRAW_BLOCKS = 148;                     // SMs; the fp32 kernel has one to three blocks on each
constexpr int DRAW_EXACT_BLOCKS = 148;               // rows of scratch in the workspace
constexpr float ROW_FLOOR = 2.384185791015625e-7f;   // 2^-22: weights that are formed again where fp32 does not do
constexpr float ROW_TAIL = 5.9604645e-8f;            // 2^-24: weights that a row of few heavy entries does without
// Rows whose largest exponent is at least this: fp32's last place of exponents shows in log probabilities, which are formed from the points
// in double where they are wanted.  Their error (rms over rms), 96 lanes of 100 x 77, d = 8, eps from 0.01: 1e-5 without, 4e-7 from
// 48 on (11 us more), 1e-7 from 16 on.  2 lanes of 8192 x 8192, d = 3: 613 us and 8e-7 without, 768 us and 4e-8 so.  From 16 on
// rows of exponents of some tens take part, too: 256 lanes of 512 x 512, d = 15, threefold the time (twofold with heavy entries alone, below), for
// 2e-7 without.
constexpr float DRAW_FAR = 48.f;
// Deep rows lose as much from smaller exponents on, (d + 6) 2^-24 of them.  Up to 48 only what counts is formed again, entries above a sixteenth of the
// row and those drawn: 8 lanes of 144 x 739, d = 128, exponents of some 40: error 1.7e-6 without, 1.5e-7 so; 8 lanes of 1024 x 1024, d = 128,
// exponents of some 29, of which those above 30 take part: 612 us, 524 without; half the limit 721, and with all entries 1950.
constexpr float DRAW_FAR_SUMS = 4096.f;
// Products that are held at a time.  64 lanes of 1024 x 1024 x 512: 843 us by 64 MB, which stay in the L2 cache, 780 by 128 MB,
// 743 all at once (with products of one accumulator; 751 so now): the rows that are formed again are then one launch, too.
constexpr size_t DRAW_DOTS_BYTES = (size_t)512 << 20;

struct Draw {
    const void *x, *y;
    Cloud4 x4, y4;
    const double *g;
    const float *eps, *temperature, *top_p, *min_p, *u;
    const int *top_k;
    const int *status;                               // of a batch's lanes, or null
    float far;                                       // rows whose largest exponent is above have log probabilities from their points
    int *index;
    float *logp;
    int dtype, W, n, m, d, S, mp;
    // workspace
    double *hn;                                      // [W][mp] k g_j, or k (g_j - |y_j|^2); -inf: masked
    float *yt;                                       // [W][d][mp] (differences)
    float2 *yn, *xn;                                 // [W][mp], [W][n] squared norms, and their means over prefixes (products)
    const float *dots;                               // rows row0 .. row0 + rows - 1 of lanes lane0 .. lane0 + lanes - 1
    double *scratch;                                 // [blocks][mp] weights of rows in float64
    long long *list;                                 // rows that are open: their number, then which; null: all rows
    unsigned *later_n;                               // products: rows of this launch that are formed again by a launch of
    long long *later;                                // their own, their number and which; null: formed again at once
    int launches;                                    // numbers that later_n has, one for each launch
    long long ldo;
    int lane0, lanes, row0, rows;
};

struct Lane {
    RowCuts cuts;
    double k2;
    bool ok;
};
__device__ __forceinline__ Lane lane_of(const Draw &P, int w)
{
    Lane L;
    float T = P.temperature ? P.temperature[w] : 1.f;
    int k = P.top_k ? P.top_k[w] : 0;
    const float p = P.top_p ? P.top_p[w] : 1.f, r = P.min_p ? P.min_p[w] : 0.f, eps = P.eps[w];
    L.ok = T >= 0.f && T <= 3.402823466e38f && k >= 0 && p > 0.f && r >= 0.f && r <= 1.f && eps > 0.f && eps <= 3.402823466e38f;
    if (T == 0.f) { T = 1.f; k = 1; }
    L.cuts.k = k == 0 ? INT_MAX : k;
    L.cuts.p = (double)p;
    L.cuts.r = r;
    L.k2 = 1.4426950408889634 / ((double)eps * (double)T);
    return L;
}
__device__ __noinline__ float raw_value(const void *base, const Cloud4 &c, int dtype, size_t row, int d, int k)
{
    if (dtype == SKB_F32) return ((const float *)base)[row * d + k];
    if (dtype == SKB_BF16) return __uint_as_float((uint32_t)((const uint16_t *)base)[row * d + k] << 16);
    return cloud4_value(c, row, k);
}
// A lane that its batch gave up has potentials that mean nothing: NaN in the place of all k g, which closes its rows.  (The settings'
// check would be the place to ask; there it costs the kernel of rows by warps 43 of 686 us.)
__device__ __forceinline__ bool given_up(const Draw &P, int w) { return P.status && P.status[w] == SKB_LANE_NONFINITE; }
// Transposed copy of y and k g, 32 points to a block.  Masked points get coordinates of zero, whatever theirs are.
__global__ void __launch_bounds__(256) transpose_kernel(const __grid_constant__ Draw P)
{
    __shared__ float tile[32][33];
    __shared__ int masked[32];
    const int w = blockIdx.y, j0 = blockIdx.x * 32, tid = threadIdx.x, col = tid & 31, part = tid >> 5;
    const Lane L = lane_of(P, w);
    if (P.list && blockIdx.x == 0 && w == 0 && tid == 0) P.list[0] = 0;
    if (tid < 32) {
        const int j = j0 + tid;
        const double g = j < P.m ? P.g[(size_t)w * P.m + j] : -CUDART_INF;
        masked[tid] = g == -CUDART_INF;
        if (j < P.mp) P.hn[(size_t)w * P.mp + j] = given_up(P, w) ? CUDART_NAN : g == -CUDART_INF ? g : L.k2 * g;
    }
    __syncthreads();
    float *yt = P.yt + (size_t)w * P.d * P.mp;
    if (P.d <= 8) {
        if (part < P.d) yt[(size_t)part * P.mp + j0 + col] = masked[col] ? 0.f : raw_value(P.y, P.y4, P.dtype, (size_t)w * P.m + j0 + col, P.d, part);
        return;
    }
#pragma unroll 1
    for (int k0 = 0; k0 < P.d; k0 += 32) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int j = part + 8 * q, k = k0 + col;
            tile[j][col] = k < P.d && !masked[j] ? raw_value(P.y, P.y4, P.dtype, (size_t)w * P.m + j0 + j, P.d, k) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int k = k0 + part + 8 * q;
            if (k < P.d) yt[(size_t)k * P.mp + j0 + col] = tile[col][part + 8 * q];
        }
        __syncthreads();
    }
}

// Eight dimensions of a point from k on, k a multiple of 8, as they are held (loads of many of these are in flight
// before the first is looked at): bf16, or codes and their scale's byte.
struct Eight { uint4 a; };
template <bool BF>
__device__ __forceinline__ Eight load_eight(const void *data, const Cloud4 &c, size_t row, int d, int k)
{
    Eight e;
    if constexpr (BF) e.a = *reinterpret_cast<const uint4 *>((const uint16_t *)data + row * d + k);
    else {
        e.a.x = *reinterpret_cast<const uint32_t *>(c.codes + row * c.cb + k / 2);
        e.a.y = c.scales[row * c.sb + (c.points ? k >> 4 : k >> 5)];
    }
    return e;
}
// `point`: the point's power of two (nv4)
template <bool BF>
__device__ __forceinline__ void eight_values(const Eight &e, const Cloud4 &c, float point, float (&v)[8])
{
    if constexpr (BF) {
        const uint32_t b[4] = {e.a.x, e.a.y, e.a.z, e.a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(b[i] << 16); v[2 * i + 1] = __uint_as_float(b[i] & 0xffff0000u); }
    } else {
        const float s = c.points ? e4m3_value(e.a.y) * point : e8m0_value(e.a.y);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = e2m1_value(e.a.x >> (4 * i)) * s;
    }
}
__host__ __device__ inline int dots_xd(int d) { return (d + 31) / 32 * 32; }
// |point|^2 in float64, by one warp; prefix: the mean, over steps of 16 dimensions, of the squared norm of what the
// accumulator has seen of the point by then (bf16: accumulators begin anew every DOTS_BF16_PART dimensions).
template <bool BF>
__device__ __forceinline__ double square_of(const void *base, const Cloud4 &c, size_t row, int d, double &prefix)
{
    double s = 0.0;
    float p = 0.f;
    const int steps = (d + 15) / 16, chunks = BF ? d / 8 : dots_xd(d) / 8;
    const float point = !BF && c.points ? c.points[row] : 1.f;
#pragma unroll 2
    for (int q = threadIdx.x & 31; q < chunks; q += 32) {
        float v[8], f = 0.f;
        eight_values<BF>(load_eight<BF>(base, c, row, d, 8 * q), c, point, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // (in double: the square of a value beyond 2^64 is infinite in fp32, and a norm that is infinite would mask its target)
            s = fma((double)v[i], (double)v[i], s);
            f = fmaf(v[i], v[i], f);
        }
        const int until = BF ? min(steps, (8 * q / DOTS_BF16_PART + 1) * (DOTS_BF16_PART / 16)) : steps;
        p = fmaf(f, (float)max(until - q / 2, 1), p);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, off);
        p += __shfl_xor_sync(0xffffffffu, p, off);
    }
    prefix = (double)(p / (float)steps) * 1.00001;                   // (the roundings of p)
    return s;
}
// k (g - |y|^2), and what bounds the error of the products, a warp to a point.
template <bool BF>
__global__ void __launch_bounds__(256) norms_kernel(const __grid_constant__ Draw P)
{
    const int w = blockIdx.y, i = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    double p = 0.0;
    if (blockIdx.x == 0 && w == 0) {
        if (threadIdx.x == 0) P.list[0] = 0;
#pragma unroll 1
        for (int q = threadIdx.x; q < P.launches; q += 256) P.later_n[q] = 0u;
    }
    if (i < P.mp) {
        const double g = i < P.m ? P.g[(size_t)w * P.m + i] : -CUDART_INF;
        const bool masked = g == -CUDART_INF;
        const double s = masked ? 0.0 : square_of<BF>(P.y, P.y4, (size_t)w * P.m + i, P.d, p);
        if (lane == 0) {
            P.hn[(size_t)w * P.mp + i] = given_up(P, w) ? CUDART_NAN : masked ? g : lane_of(P, w).k2 * (g - s);
            P.yn[(size_t)w * P.mp + i] = make_float2((float)s, (float)p);
        }
        return;
    }
    const int r = i - P.mp;
    if (r >= P.n) return;
    const double s = square_of<BF>(P.x, P.x4, (size_t)w * P.n + r, P.d, p);
    if (lane == 0) P.xn[(size_t)w * P.n + r] = make_float2((float)s, (float)p);
}

__device__ __forceinline__ void put_draw(const Draw &P, size_t at, int index, float logp)
{
    P.index[at] = index;
    if (P.logp) P.logp[at] = logp;
}

// Draws of one row from `len` weights, of columns `where` (null: their places), and their cut, shared out to the group's warps.  True if all of this warp's were sure.
template <typename Real>
__device__ __noinline__ bool draw_all(const Draw &P, size_t row, const Real *w, int len, const unsigned short *where, const RowCut<Real> &cut, const double *tiles, const RowError &err, int warp, int warps)
{
    const double total = row_total(tiles, len / ROW_TILE);
    bool sure = true;
#pragma unroll 1
    for (int s = warp; s < P.S; s += warps) {
        const float u = P.u[row * P.S + s];
        int j = -1;
        double wj = 0.0;
        if (u >= 0.f && u < 1.f) {
            const bool good = row_draw(w, cut, tiles, len / ROW_TILE, total, (double)u, err, j, wj);
            if (!good) { sure = false; continue; }
        }
        if ((threadIdx.x & 31) == 0) put_draw(P, row * P.S + s, where && j >= 0 ? where[j] : j, j < 0 ? CUDART_NAN_F : (float)log(wj / total));
    }
    return sure;
}
__device__ __noinline__ void draw_none(const Draw &P, size_t row, int t, int nt)
{
#pragma unroll 1
    for (int s = t; s < P.S; s += nt) put_draw(P, row * P.S + s, -1, CUDART_NAN_F);
}


// Exponents of a row from the points as they are held, eight threads to a point, four points to a warp.
constexpr int BATCH = 8;                             // loads in flight
template <bool BF>
__device__ __forceinline__ void exact_rows(const Draw &P, const Lane &L, int w, const double *hn, const double *xs, double *wd, int warp, int warps,
                                           double &top, int &bad)
{
    const int lane = threadIdx.x & 31, part = lane & 7, chunks = BF ? P.d / 8 : dots_xd(P.d) / 8, rounds = (chunks + 7) / 8, d = P.d;
    const void *y_data = P.y;
    const Cloud4 y4 = P.y4;
    const int eights = dots_xd(d) / 8;               // (x is kept as [8][d / 8]: threads next to each other read next to each other)
#pragma unroll 1
    for (int j0 = 4 * warp; j0 < P.mp; j0 += 4 * warps) {
        const int j = j0 + (lane >> 3);
        const bool is = hn[j] != -CUDART_INF;
        double c = 0.0;
        if (is) {
            const size_t row = (size_t)w * P.m + j;
            const float point = !BF && y4.points ? y4.points[row] : 1.f;
#pragma unroll 1
            for (int r0 = 0; r0 < rounds; r0 += BATCH) {
                Eight y8[BATCH];
#pragma unroll
                for (int b = 0; b < BATCH; ++b)
                    if (r0 + b < rounds) y8[b] = load_eight<BF>(y_data, y4, row, d, 8 * min(8 * (r0 + b) + part, chunks - 1));
#pragma unroll
                for (int b = 0; b < BATCH; ++b)
                    if (r0 + b < rounds) {
                        const int q = 8 * (r0 + b) + part;
                        float y[8];
                        double sum = 0.0;
                        eight_values<BF>(y8[b], y4, point, y);
#pragma unroll
                        for (int i = 0; i < 8; ++i) { const double f = xs[i * eights + min(q, chunks - 1)] - (double)y[i]; sum = fma(f, f, sum); }
                        if (q < chunks) c += sum;
                    }
            }
        }
#pragma unroll
        for (int off = 1; off < 8; off *= 2) c += __shfl_xor_sync(0xffffffffu, c, off);
        const double z = is ? L.k2 * (P.g[(size_t)w * P.m + j] - c) : -CUDART_INF;
        if (part == 0) wd[j] = z;
        top = fmax(top, z);
        bad |= !(z <= 1.7e308);
    }
}

// Rows in float64, a block to a row: those of the list, or all (rows too long for shared memory).
__global__ void __launch_bounds__(512) draw_exact_kernel(const __grid_constant__ Draw P)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowScratch sc;
    double *tiles = reinterpret_cast<double *>(smem), *xs = tiles + P.mp / ROW_TILE, *wd = P.scratch + (size_t)blockIdx.x * P.mp;
    const int tid = threadIdx.x, nt = blockDim.x, warp = tid >> 5, xd = dots_xd(P.d);
    const RowGroup G = {tid, nt, 0, &sc};
    const long long rows = P.list ? P.list[0] : (long long)P.W * P.n;
#pragma unroll 1
    for (long long t = blockIdx.x; t < rows; t += gridDim.x) {
        const long long row = P.list ? P.list[1 + t] : t;
        const int w = (int)(row / P.n);
        const Lane L = lane_of(P, w);
        const double *hn = P.hn + (size_t)w * P.mp;
        __syncthreads();
        if (!L.ok) { draw_none(P, (size_t)row, tid, nt); continue; }
#pragma unroll 1
        for (int k = tid; k < xd; k += nt)
            xs[P.yt ? k : (k & 7) * (xd / 8) + (k >> 3)] = k < P.d ? (double)raw_value(P.x, P.x4, P.dtype, (size_t)row, P.d, k) : 0.0;
        __syncthreads();
        double top = -CUDART_INF;
        int bad = 0;
        if (P.yt) {
            const float *yt = P.yt + (size_t)w * P.d * P.mp;
#pragma unroll 1
            for (int j = tid; j < P.mp; j += nt) {
                double c = 0.0;
#pragma unroll 4
                for (int k = 0; k < P.d; ++k) {
                    const double e = xs[k] - (double)yt[(size_t)k * P.mp + j];
                    c = fma(e, e, c);
                }
                const double z = hn[j] == -CUDART_INF ? -CUDART_INF : fma(-L.k2, c, hn[j]);
                wd[j] = z;
                top = fmax(top, z);
                bad |= !(z <= 1.7e308);
            }
        } else {
            if (P.dtype == SKB_BF16) exact_rows<true>(P, L, w, hn, xs, wd, warp, nt >> 5, top, bad);
            else exact_rows<false>(P, L, w, hn, xs, wd, warp, nt >> 5, top, bad);
        }
        double mass = 0.0;
        int count = 0;
        top = G.largest(top);
        G.add(mass, bad);                                           // (a barrier: wd is written)
        if (bad || top == -CUDART_INF) { draw_none(P, (size_t)row, tid, nt); continue; }
#pragma unroll 1
        for (int j = tid; j < P.mp; j += nt) {
            const double v = exp2(wd[j] - top);
            wd[j] = v;
            mass += v;
            count += v > 0.0;
        }
        G.add(mass, count);
        const RowError none = {0.0, 0.f, 0.f};
        RowCut<double> cut;
        row_cut(wd, P.mp, G, L.cuts, 1.0, mass, count, none, cut, tiles);
        draw_all(P, (size_t)row, wd, P.mp, nullptr, cut, tiles, none, warp, nt >> 5);
        __syncthreads();
    }
}

// Rows in fp32: a row's exponents, then weights, in shared memory, by a warp or a group of warps each.  h: the lane's hn less its
// largest; xs: -x, twice each (differences), or x of a row that is formed again (products).
// Error of an exponent t = log2 w at a depth q below the row's largest, A = |largest t|:
//   differences  h <= 0 and the scaled distance h - t are at most A + q; d + 2 roundings of the distance, three of the
//                scale and t, one of h: (d + 6) (A + q) 2^-24
//   products     2 k |x . y| is at most B = 2 k |x| max |y|, and what an accumulator has seen of it after each 16 dimensions at most the
//                same of those dimensions, on average no more than B' (from the root mean squares of their norms).  The matrix unit
//                cuts off (skb_dots.cu): bf16, for 16 dimensions, 16 products and the sum so far at 2^-25 of the largest and the
//                result to 24 bits, 17 / 4 + 1 units of 2^-23 of that; 4-bit kinds, for 64 dimensions, four blocks of a scale
//                and the sum, 5 / 4 + 1 units, counted as 4.  (d / 16) (5.25 or 1) B' 2^-23, the additions of bf16's parts
//                B 2^-24 each; the roundings of h, scale and t: (3 B + 3 (A + q)) 2^-24
// The exponential adds 2^-22 and 2^-24 q of the difference that it is taken of, the additions of weights 2^-24 each.
// Mass, number and largest of a row's weights, and the mass of those at most ROW_FLOOR.
struct RowSums {
    double mass, rest;
    int count;
    float top;
};
__device__ __forceinline__ RowSums sum_row(const RowGroup &G, const float *w, int mp)
{
    RowSums r = {0.0, 0.0, 0, 0.f};
#pragma unroll 1
    for (int j = 4 * G.t; j < mp; j += 4 * G.nt) {
        float v[4];
        load4(w + j, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double d = (double)v[i];
            r.mass += d;
            r.rest += v[i] > ROW_FLOOR ? 0.0 : d;
            r.count += v[i] > 0.f;
            r.top = fmaxf(r.top, v[i]);
        }
    }
    int unused = 0;
    G.add(r.mass, r.count);
    G.add(r.rest, unused);
    r.top = G.largest(r.top);
    return r;
}

// Exact weights, to fp32's precision, for a row's entries above 2^-22, by a warp for its tiles' entries of the row
// (tiles warp, warp + warps, ...).  `base`: what an exponent of h stands for in float64, the row's largest included.
__device__ __forceinline__ void refine_differences(const Draw &P, double k2, const double *hn, const float *yt, const float *nx, int step, double base,
                                                   float *w, int warp, int warps)
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int q = warp; q < P.mp / ROW_TILE; q += warps) {
        const int j = q * ROW_TILE + 4 * lane;
        float v[4];
        load4(w + j, v);
        if (!(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])) > ROW_FLOOR)) continue;
        double c[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 1
        for (int k = 0; k < P.d; ++k) {
            float y[4];
            load4(yt + (size_t)k * P.mp + j, y);
            const double x = (double)nx[k * step];
#pragma unroll
            for (int i = 0; i < 4; ++i) { const double e = (double)y[i] + x; c[i] = fma(e, e, c[i]); }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (v[i] > ROW_FLOOR) v[i] = (float)exp2(fma(-k2, c[i], hn[j + i]) - base);
        *reinterpret_cast<float4 *>(w + j) = make_float4(v[0], v[1], v[2], v[3]);
    }
}
// x . y of four points of y at a time, eight threads to a point.  Products are exact in fp32 (at most 16 bits).  They are
// added to a large number M, whose last place is 2^-24 of a bound on the sum: what an addition cuts off is itself exact and is
// added up apart, so that the result is good to 2^-40 of the bound.
template <bool BF>
__device__ __forceinline__ void refine_products(const Draw &P, double k2, int wl, const double *hn, const float *x, float magic, double base, float *w,
                                                int len, const unsigned short *where, int count, unsigned char *bytes, int warp, int warps)
{
    const int lane = threadIdx.x & 31, part = lane & 7, col = lane >> 3;
    const int chunks = BF ? P.d / 8 : dots_xd(P.d) / 8, rounds = (chunks + 7) / 8, m = P.m, d = P.d;
    const void *y_data = P.y;
    const Cloud4 y4 = P.y4;
    // (a list: its entries shared out among all warps; a row: its tiles)
    const int first = where ? 4 * warp : 0, step = where ? 4 * warps : 4;
#pragma unroll 1
    for (int q = where ? 0 : warp; q < len / ROW_TILE; q += where ? 1 : warps) {
        int n = 0;
        if (where) n = min(ROW_TILE, count - q * ROW_TILE);
        else {
            float v[4];
            load4(w + q * ROW_TILE + 4 * lane, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned ball = __ballot_sync(0xffffffffu, v[i] > ROW_FLOOR);
                if (v[i] > ROW_FLOOR) bytes[n + __popc(ball & ((1u << lane) - 1u))] = (unsigned char)(4 * lane + i);
                n += __popc(ball);
            }
            __syncwarp();
        }
#pragma unroll 1
        for (int e0 = first; e0 < n; e0 += step) {
            const int e = min(e0 + col, n - 1), at = q * ROW_TILE + (where ? e : bytes[e]), j = where ? where[at] : at;
            const size_t row = (size_t)wl * m + j;
            const float point = !BF && y4.points ? y4.points[row] : 1.f;
            const u64 m2 = pack2(magic, magic);
            const double hj = hn[j];
            u64 sum = m2, low = 0ull;
#pragma unroll 1
            for (int r0 = 0; r0 < rounds; r0 += BATCH) {
                Eight y8[BATCH];
#pragma unroll
                for (int b = 0; b < BATCH; ++b)
                    if (r0 + b < rounds) y8[b] = load_eight<BF>(y_data, y4, row, d, 8 * min(8 * (r0 + b) + part, chunks - 1));
#pragma unroll
                for (int b = 0; b < BATCH; ++b)
                    if (r0 + b < rounds) {
                        const int c = 8 * (r0 + b) + part;
                        float y[8];
                        eight_values<BF>(y8[b], y4, point, y);
                        const ulonglong2 *xp = reinterpret_cast<const ulonglong2 *>(x + 8 * min(c, chunks - 1));
                        u64 xv[4] = {xp[0].x, xp[0].y, xp[1].x, xp[1].y};
                        if (c >= chunks) xv[0] = xv[1] = xv[2] = xv[3] = 0ull;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const u64 yv = pack2(y[2 * i], y[2 * i + 1]), t = fma2(xv[i], yv, sum);
                            low = add2(low, fma2(xv[i], yv, sub2(sum, t)));
                            sum = t;
                        }
                    }
            }
            float a, b, la, lb;
            unpack2(sub2(sum, m2), a, b);                            // exact
            unpack2(low, la, lb);
            double dot = ((double)a + (double)b) + ((double)la + (double)lb);
#pragma unroll
            for (int off = 1; off < 8; off *= 2) dot += __shfl_xor_sync(0xffffffffu, dot, off);
            if (part == 0 && e0 + col < n) w[at] = (float)exp2(fma(2.0 * k2, dot, hj) - base);
        }
        __syncwarp();
    }
}
// The same from differences, for a list of entries, one to a thread.
__device__ __forceinline__ void refine_list(const Draw &P, double k2, const double *hn, const float *yt, const float *nx, int step, double base, float *w,
                                            const unsigned short *where, int n, int t, int nt)
{
#pragma unroll 1
    for (int q = t; q < n; q += nt) {
        const int j = where[q];
        double c = 0.0;
#pragma unroll 4
        for (int k = 0; k < P.d; ++k) {
            const double e = (double)yt[(size_t)k * P.mp + j] + (double)nx[k * step];
            c = fma(e, e, c);
        }
        w[q] = (float)exp2(fma(-k2, c, hn[j]) - base);
    }
}

// log2 of an entry's weight where the row's largest has 2^base, from its points in double.
__device__ __forceinline__ float exact_gap(const Draw &P, double k2, int wl, const float *nx, int step, double base, int j)
{
    const float *yt = P.yt + (size_t)wl * P.d * P.mp + j;
    const double h = P.hn[(size_t)wl * P.mp + j];
    double c = 0.0;
#pragma unroll 4
    for (int k = 0; k < P.d; ++k) {
        const double e = (double)yt[(size_t)k * P.mp] + (double)nx[k * step];
        c = fma(e, e, c);
    }
    return (float)(fma(-k2, c, h) - base);
}
// Log probabilities of a row's draws once more, heavy entries from their points; w: weights, kept from tau on; A: the largest exponent.  Heavy
// are those above ROW_FLOOR, up to DRAW_FAR those above a sixteenth of the row (the others' errors add up to less than one's, being
// independent).  The group's last threads have the draws, so that in a group of several warps they need not wait for the sum.
__device__ __forceinline__ void exact_logs(const Draw &P, double k2, int wl, size_t row, const RowGroup &G, double base, const float *nx, int step, const float *w,
                                           int len, const unsigned short *where, float tau, float A)
{
    const int first = G.nt - 1 - G.t;
    double mass = 0.0;
    float gap = 0.f, heavy = ROW_FLOOR;
    int j = first < P.S ? P.index[row * P.S + first] : -1, unused = 0;
    if (j >= 0) gap = exact_gap(P, k2, wl, nx, step, base, j);
    if (A <= DRAW_FAR) {
        double all = 0.0;
#pragma unroll 1
        for (int q = G.t; q < len; q += G.nt) all += quick_kept(w[q], tau) ? (double)w[q] : 0.0;
        G.add(all, unused);
        heavy = fmaxf(heavy, (float)all * 0.0625f);
    }
#pragma unroll 1
    for (int q = G.t; q < len; q += G.nt) {
        float v = w[q];
        if (!quick_kept(v, tau)) continue;
        if (v > heavy) v = ex2_fast(exact_gap(P, k2, wl, nx, step, base, where ? where[q] : q));
        mass += (double)v;
    }
    G.add(mass, unused);
    const float whole = log2f((float)mass);
#pragma unroll 1
    for (int s = first; s < P.S;) {
        if (j >= 0) P.logp[row * P.S + s] = 0.69314718f * (gap - whole);
        if ((s += G.nt) >= P.S) break;
        j = P.index[row * P.S + s];
        if (j >= 0) gap = exact_gap(P, k2, wl, nx, step, base, j);
    }
}

// Sums over the group of three floats and a count, in one order; `before`: of the count over the warps before this one.
__device__ __forceinline__ void group_sums(const RowGroup &G, float (&f)[3], unsigned &n, unsigned &before, int &turn)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
#pragma unroll
        for (int i = 0; i < 3; ++i) f[i] += __shfl_xor_sync(0xffffffffu, f[i], off);
    n = __reduce_add_sync(0xffffffffu, n);
    before = 0;
    if (G.nt == 32) return;
    turn ^= 1;
    if ((G.t & 31) == 0) {
        unsigned *p = G.sc->part[turn][G.t >> 5];
#pragma unroll
        for (int i = 0; i < 3; ++i) p[i] = __float_as_uint(f[i]);
        p[3] = n;
    }
    G.sync();
    f[0] = f[1] = f[2] = 0.f;
    n = 0;
#pragma unroll 1
    for (int q = 0; q < G.nt >> 5; ++q) {
        const unsigned *p = G.sc->part[turn][q];
#pragma unroll
        for (int i = 0; i < 3; ++i) f[i] += __uint_as_float(p[i]);
        if (q < G.t >> 5) before += p[3];
        n += p[3];
    }
}
__device__ __forceinline__ float group_largest(const RowGroup &G, float v, int &turn)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
    if (G.nt == 32) return v;
    turn ^= 1;
    if ((G.t & 31) == 0) G.sc->part[turn][G.t >> 5][0] = __float_as_uint(v);
    G.sync();
#pragma unroll 1
    for (int q = 0; q < G.nt >> 5; ++q) v = fmaxf(v, __uint_as_float(G.sc->part[turn][q][0]));
    return v;
}
// Whether all warps of the group say so.
__device__ __forceinline__ bool group_all(const RowGroup &G, bool v, int &turn)
{
    v = __all_sync(0xffffffffu, v);
    if (G.nt == 32) return v;
    turn ^= 1;
    if ((G.t & 31) == 0) G.sc->part[turn][G.t >> 5][0] = v;
    G.sync();
#pragma unroll 1
    for (int q = 0; q < G.nt >> 5; ++q) v = v && G.sc->part[turn][q][0] != 0;
    return v;
}

// A row once more: what weighs more than ROW_FLOOR to fp32's last place, what does not is `off` of itself off.  x: -x, `step`
// apart (differences), or room for a row (products), whose bound is `bound` (differences: the row's largest exponent).  A row that is a list of n entries, columns
// `where`, has a mass `tail` besides; `loose` is the mass of entries among which a cut was left out.  A row of which only the
// logarithms are to be formed again has its cut in `tau`, the others a negative one.
template <bool DOTS>
__device__ __noinline__ bool again(const Draw &P, double k2, RowCuts cuts, int wl, size_t row, const RowGroup &G, double base, float off, float bound, float *x,
                                   int step, float *w, int len, const unsigned short *where, int n, float tail, float loose, double *tiles, unsigned char *bytes, float tau)
{
    const double *hn = P.hn + (size_t)wl * P.mp;
    if (!DOTS && tau >= 0.f) {
        exact_logs(P, k2, wl, row, G, base, x, step, w, len, where, tau, bound);
        return true;
    }
    if (DOTS) {
        const int xd = dots_xd(P.d);
#pragma unroll 1
        for (int k = G.t; k < xd; k += G.nt) x[k] = k < P.d ? raw_value(P.x, P.x4, P.dtype, row, P.d, k) : 0.f;
        // twice to four times the bound, and half as much again: sums within the bound stay in its binade
        const float magic = 1.5f * __uint_as_float((__float_as_uint(bound * 4.f) & 0x7f800000u) + 0x00800000u);
        G.sync();
        if (P.dtype == SKB_BF16) refine_products<true>(P, k2, wl, hn, x, magic, base, w, len, where, n, bytes, G.t >> 5, G.nt >> 5);
        else refine_products<false>(P, k2, wl, hn, x, magic, base, w, len, where, n, bytes, G.t >> 5, G.nt >> 5);
    } else if (where) refine_list(P, k2, hn, P.yt + (size_t)wl * P.d * P.mp, x, step, base, w, where, n, G.t, G.nt);
    else refine_differences(P, k2, hn, P.yt + (size_t)wl * P.d * P.mp, x, step, base, w, G.t >> 5, G.nt >> 5);
    G.sync();
    const RowSums sums = sum_row(G, w, len);
    if (!(sums.mass <= 3e38)) return false;
    // (a list's entries are all formed again; what is not in it counts in the row's mass, of which a cut takes its share, and is
    // missing from the sums that are drawn from where there is no cut)
    RowError fine = {2.0 * (5.9604645e-8 * sums.mass + (where ? (double)tail : sums.rest) * off), 2.f * 5.9604645e-8f, 0.f};
    // a share is of what the ranks left: where their cut was left out, of up to `loose` less
    RowError edge = fine;
    if (cuts.p < 1.0) edge.sums += 1.04 * (double)loose;
    RowCut<float> cut;
    if (!row_cut(w, len, G, cuts, sums.top, sums.mass + (double)tail, sums.count, edge, cut, tiles) || cut.lowest < 2.f * ROW_FLOOR) return false;
    fine.sums += 2.04 * (double)(cut.tau == 0.f ? fmaxf(tail, loose) : loose);
    return draw_all(P, row, w, len, where, cut, tiles, fine, G.t >> 5, G.nt >> 5);
}

// What the rows of a lane have in common, and a group's room in shared memory.
struct LaneState {
    Lane L;
    int lane;
    double h_top;
    float k2, p, y_max, y_prefix;
    bool some;
};
struct RowRoom {
    float *w;                    // [mp]
    double *tiles;               // [mp / 128]
    float *list;                 // [list_room(mp) + ROW_TILE] weights, and their columns
    unsigned short *where;
    float *x;                    // differences: -x, `step` apart; products: room for a row
    int step;
    unsigned char *bytes;        // of this warp, [128] (products)
};
__host__ __device__ inline int list_room(int mp) { return (mp / 4 + ROW_TILE - 1) / ROW_TILE * ROW_TILE; }

// Settings of lane `lane`, its largest k g_j (- |y_j|^2), and the others less that; by all threads, NT of them.
template <int NT, bool DOTS>
__device__ __forceinline__ void enter_lane(const Draw &P, LaneState &S, int lane, float *h, const RowGroup &all)
{
    __syncthreads();
    S.lane = lane;
    S.L = lane_of(P, lane);
    // Distances past fp32's range are as good as infinite beside k from 1e-34 on (a row is decided in fp32 while its largest exponent is below
    // 34000; 1e-34 times 3.4e38 is as much), and what is lost below the range is nothing up to 1e27 (2 k d 2^-126 < 2^-25 of an exponent).
    // Other lanes' exponents are NaN in fp32, which leaves their rows to float64.
    S.k2 = S.L.k2 >= 1e-34 && S.L.k2 <= 1e27 ? (float)S.L.k2 : CUDART_NAN_F;
    S.p = (float)S.L.cuts.p;
    const double *hn = P.hn + (size_t)lane * P.mp;
    double top = -CUDART_INF;
    float far = 0.f, prefix = 0.f;
#pragma unroll 1
    for (int j = threadIdx.x; j < P.mp; j += NT) {
        top = fmax(top, hn[j]);
        if (DOTS) {
            const float2 s = P.yn[(size_t)lane * P.mp + j];
            far = fmaxf(far, s.x);
            prefix = fmaxf(prefix, s.y);
        }
    }
    S.h_top = all.largest(top);
    if (DOTS) { S.y_max = sqrtf(all.largest(far)); S.y_prefix = sqrtf(all.largest(prefix)); }
    S.some = S.L.ok && S.h_top != -CUDART_INF;
#pragma unroll 1
    for (int j = threadIdx.x; j < P.mp; j += NT) h[j] = S.some ? (float)(hn[j] - S.h_top) : 0.f;
    __syncthreads();
}

// One row by its group: exponents (in w for differences, to be formed from `dots` for products) to weights, cut, draws.
// LATER: a row that is to be formed again goes on a list.
template <bool DOTS, bool LATER>
__device__ __forceinline__ void do_row(const Draw &P, const LaneState &S, size_t row, const RowGroup &G, int &turn, const RowRoom &M, const float *h,
                                       const float *dots)
{
    constexpr float u24 = 5.9604645e-8f;
    const int mp = P.mp, ntiles = mp / ROW_TILE, lane = G.t & 31;
    float *w = M.w;
    unsigned *units = reinterpret_cast<unsigned *>(M.tiles);     // (never at the same time)
    const Span span(G, mp);
    const float u_first = P.u[row * P.S];
    float2 xn = make_float2(0.f, 0.f);
    float top = -CUDART_INF_F;
    if (DOTS) {
        xn = P.xn[row];
        const float two_k = 2.f * S.k2;
#pragma unroll 1
        for (int j0 = span.begin; j0 < span.end; j0 += 8 * span.step) {
            float4 d[8];
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (j0 + q * ROW_TILE < span.end) d[q] = *reinterpret_cast<const float4 *>(dots + j0 + q * ROW_TILE);
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (j0 + q * ROW_TILE < span.end) {
                    float v[4] = {d[q].x, d[q].y, d[q].z, d[q].w}, hh[4];
                    load4(h + j0 + q * ROW_TILE, hh);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[i] = hh[i] == -CUDART_INF_F ? -CUDART_INF_F : fmaf(two_k, v[i], hh[i]);
                        top = fmaxf(top, v[i]);
                    }
                    *reinterpret_cast<float4 *>(w + j0 + q * ROW_TILE) = make_float4(v[0], v[1], v[2], v[3]);
                }
        }
    } else {
#pragma unroll 4
        for (int j = span.begin; j < span.end; j += span.step) {
            float v[4];
            load4(w + j, v);
            top = fmaxf(fmaxf(top, fmaxf(v[0], v[1])), fmaxf(v[2], v[3]));
        }
    }
    top = group_largest(G, top, turn);
    // nothing left in fp32's range, a NaN or an infinite exponent: float64 tells which
    bool sure = false;
    if (top != -CUDART_INF_F) {
        float f[3] = {0.f, 0.f, 0.f};                            // mass, sum of w log2(1 / w), mass below ROW_TAIL
        unsigned heavy = 0, before, has = 0, bit = 1;            // has: this thread's tiles with a heavy entry (the first 32)
#pragma unroll 4
        for (int j = span.begin; j < span.end; j += span.step) { // (each thread's own: no barrier yet)
            float v[4];
            load4(w + j, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float gap = v[i] - top, down = gap < -200.f ? -200.f : gap;    // (2^-200 is zero already; a NaN stays)
                v[i] = ex2_fast(down);
                f[1] = fmaf(-down, v[i], f[1]);
                if (v[i] >= ROW_TAIL) { ++heavy; has |= bit; }
                else f[2] += v[i];
            }
            bit <<= 1;
            *reinterpret_cast<float4 *>(w + j) = make_float4(v[0], v[1], v[2], v[3]);
            f[0] += (v[0] + v[1]) + (v[2] + v[3]);
        }
        group_sums(G, f, heavy, before, turn);
        G.sync();
        const float mass = f[0];
        if (mass <= 3e38f) {
            const float k2 = S.k2, A = fabsf(top);
            float fixed, slope, bound = 0.f;                     // of an exponent: fixed + slope q
            if (DOTS) {
                bound = sqrtf(xn.x) * S.y_max;
                slope = 3.f * u24;
                const float steps = (float)((P.d + 15) / 16), cut_off = P.dtype == SKB_BF16 ? 10.5f : 2.f,
                            joins = P.dtype == SKB_BF16 ? (float)((P.d - 1) / DOTS_BF16_PART) : 0.f;
                fixed = u24 * (2.f * k2 * (cut_off * steps * sqrtf(xn.y) * S.y_prefix + (3.f + joins) * bound) + 3.f * A);
            } else {
                slope = (float)(P.d + 6) * u24;
                fixed = slope * A;
            }
            fixed = 0.6932f * fixed + 2.4e-7f;
            slope = 0.6932f * (slope + u24);
            const RowError err = {1.0, 2.f * fixed, 2.f * slope};    // of two weights: twice the error of one
            const float off = fixed + 24.f * slope;
            if (off < 0.01f) {
                const float unit = QUICK_ONE / mass;
                // Additions, 2^-24 of a sum for each that a weight goes through.  Of the mass, which the unit is made from: a thread's
                // quadruples, 2 in each, 5 in the warp, one a warp.  A part that a cut compares: one for each of a thread's
                // weights, at most 32 in a list of the last; 3 for the unit, for its reciprocal and for the product.  A draw's
                // sums, parts and whole, are of the same unit: 3 and the product, twice.  Roundings to units: half of one
                // for each thread of a cut's passes, of which two are joined; for each of 32 in a draw's tiles, parts and whole.
                const int warps = G.nt >> 5, quads = (ntiles + warps - 1) / warps;
                const float cuts_sums = 64.f * (float)(quads + 7 + warps + 3 + max(4 * quads, 32)) + (float)G.nt;
                QuickSlack slack = {1.02f * fixed * QUICK_ONE, slope * f[1] / mass * QUICK_ONE + (float)(64 * 8 + 32 * ntiles)};
                // Cuts among what weighs less than ROW_TAIL together make no difference that a draw could show but one inside
                // of the bounds, to which that weight is added.
                int k = S.L.cuts.k;
                float r_min = S.L.cuts.r, loose = 0.f;
                if (f[2] * 1048576.f <= mass && ((k != INT_MAX && (unsigned)k >= heavy) || (r_min > 0.f && r_min < ROW_TAIL))) {
                    if ((unsigned)k >= heavy) k = INT_MAX;
                    if (r_min < ROW_TAIL) r_min = 0.f;
                    loose = f[2];
                    slack.rest += 2.f * loose * unit;
                }
                const bool sparse = ntiles >= 4 && heavy <= (unsigned)mp / 4 && f[2] * 1048576.f <= mass;
                if (sparse) {
                    // few entries weigh anything: they are the row, by one warp, the others an error of the sums
                    slack.rest += 2.f * f[2] * unit;
                    has = (span.end - span.begin + span.step - 1) / span.step <= 32 ? __reduce_or_sync(0xffffffffu, has) : 0xffffffffu;
#pragma unroll 1
                    for (int j = span.begin, q = 0; j < span.end; j += span.step, ++q) {
                        if (!(has >> (q & 31) & 1u)) continue;
                        float v[4];
                        load4(w + j, v);
                        int c = 0, i0 = 0;
#pragma unroll
                        for (int i = 3; i >= 0; --i)
                            if (v[i] >= ROW_TAIL) { ++c; i0 = i; }
                        const unsigned one = __ballot_sync(0xffffffffu, c > 0);
                        if (!one) continue;
                        unsigned at = before + __popc(one & ((1u << lane) - 1u));
                        if (__any_sync(0xffffffffu, c > 1)) {
                            const unsigned two = __ballot_sync(0xffffffffu, c > 1), three = __ballot_sync(0xffffffffu, c > 2), four = __ballot_sync(0xffffffffu, c > 3);
                            const unsigned less = (1u << lane) - 1u;
                            at += __popc(two & less) + __popc(three & less) + __popc(four & less);
                            before += __popc(two) + __popc(three) + __popc(four);
                            unsigned to = at;
#pragma unroll
                            for (int i = 1; i < 4; ++i)
                                if (i > i0 && v[i] >= ROW_TAIL) { ++to; M.list[to] = v[i]; M.where[to] = (unsigned short)(j + i); }
                        }
                        before += __popc(one);
                        if (c) { M.list[at] = i0 == 0 ? v[0] : i0 == 1 ? v[1] : i0 == 2 ? v[2] : v[3]; M.where[at] = (unsigned short)(j + i0); }
                    }
                    const int len = (int)(heavy + ROW_TILE - 1) / ROW_TILE * ROW_TILE;
#pragma unroll 1
                    for (int j = (int)heavy + G.t; j < len; j += G.nt) M.list[j] = 0.f;
                    G.sync();
                }
                const int len = sparse ? (int)(heavy + ROW_TILE - 1) / ROW_TILE * ROW_TILE : mp;
                const float *r = sparse ? M.list : w;
                const RowGroup A1 = {sparse ? lane : G.t, sparse ? 32 : G.nt, G.bar, G.sc};
                unsigned count = heavy, own = 0;
                if (sparse) {
#pragma unroll 1
                    for (int j = 4 * lane; j < (int)heavy; j += ROW_TILE) own += (unsigned)min(4, (int)heavy - j);
                } else if (k != INT_MAX || S.p < 1.f) {
#pragma unroll 1
                    for (int j = span.begin; j < span.end; j += span.step) {
                        float v[4];
                        load4(w + j, v);
#pragma unroll
                        for (int i = 0; i < 4; ++i) own += v[i] > 0.f;
                    }
                    unsigned c[1] = {own};
                    group_add(G, c, turn);
                    count = c[0];
                }
                sure = true;
                QuickCut cut;
                cut.tau = 0.f;
                if (!sparse || G.t < 32) {
                    sure = quick_cut(r, len, A1, k, S.p, r_min, count, own, unit, slack, sparse ? fmaxf(cuts_sums, 64.f * (float)(quads + 10 + warps + len / 32) + (float)G.nt) : cuts_sums, err, M.list + (sparse ? list_room(mp) : 0),
                                     sparse ? 0u : (unsigned)list_room(mp), cut, turn);
                    if (sure) quick_tiles(r, len / ROW_TILE, A1, cut.tau, unit, units);
                }
                if (sparse && G.nt > 32) {
                    // the cut is the first warp's, the draws are everyone's
                    if (G.t == 0) { G.sc->tie_j = __float_as_int(cut.tau); G.sc->n_cand = sure; }
                    G.sync();
                    cut.tau = __int_as_float(G.sc->tie_j);
                    sure = G.sc->n_cand != 0;
                } else A1.sync();
                if (sure) {
                    const unsigned whole = quick_total(units, len / ROW_TILE);
#pragma unroll 1
                    for (int s = G.t >> 5; s < P.S; s += G.nt >> 5) {
                        const float u = s ? P.u[row * P.S + s] : u_first;
                        int j = -1;
                        float wj = 0.f;
                        if (u >= 0.f && u < 1.f && !quick_draw(r, len / ROW_TILE, cut.tau, unit, units, whole, u, slack, j, wj)) { sure = false; continue; }
                        if (lane == 0) put_draw(P, row * P.S + s, sparse && j >= 0 ? M.where[j] : j, j < 0 ? CUDART_NAN_F : logf(wj * unit / (float)whole));
                    }
                }
                sure = group_all(G, sure, turn);
                if (!sure && DOTS && LATER) {
                    if (G.t == 0) P.later[atomicAdd(P.later_n, 1u)] = (long long)row;
                    sure = true;
                } else if (!sure || (!DOTS && P.logp && A > P.far)) {
                    // once more, with better weights for what counts
                    G.sync();
                    sure = again<DOTS>(P, S.L.k2, {k, S.L.cuts.p, r_min}, S.lane, row, G, S.h_top + (double)top, off, DOTS ? bound : A, M.x, M.step, const_cast<float *>(r), len,
                                       sparse ? M.where : nullptr, (int)heavy, sparse ? f[2] : 0.f, loose, M.tiles, M.bytes, sure ? cut.tau : -1.f);
                    sure = group_all(G, sure, turn);
                }
            }
        }
    }
    if (!sure && G.t == 0) P.list[1 + (long long)atomicAdd((unsigned long long *)P.list, 1ull)] = (long long)row;
    G.sync();
}

// Rows that a warp holds: each warp for itself, RW rows at a time where exponents are formed from differences (a column's
// coordinates serve them all).  No barrier but where the lane changes, so warps need not wait for each other's rows.
constexpr int WARPS = 8;
template <int RW, bool DOTS>
struct WarpShape {
    int x, warp;                 // bytes: of a warp's points, and of all it has
    size_t all;
    __host__ __device__ WarpShape(int mp, int d)
    {
        x = DOTS ? dots_xd(d) * 4 : (RW * d * 8 + 15) / 16 * 16;
        warp = RW * mp * 4 + list_room(mp) * 6 + 2 * ROW_TILE * 4 + (mp / ROW_TILE + 1) / 2 * 16 + x;
        all = (size_t)mp * 4 + (size_t)WARPS * warp;
    }
};
template <int RW>
__device__ __forceinline__ void form_warp(const float *yt, const float *h, const u64 *xs, float *w, int mp, int d, float k2)
{
#pragma unroll 1
    for (int j = 4 * (threadIdx.x & 31); j < mp; j += ROW_TILE) {
        u64 acc[RW][2];
#pragma unroll
        for (int r = 0; r < RW; ++r) acc[r][0] = acc[r][1] = 0ull;
#pragma unroll 4
        for (int k = 0; k < d; ++k) {
            const ulonglong2 y = *reinterpret_cast<const ulonglong2 *>(yt + (size_t)k * mp + j);
#pragma unroll
            for (int r = 0; r < RW; ++r) {
                const u64 x = xs[k * RW + r], a = add2(y.x, x), b = add2(y.y, x);
                acc[r][0] = fma2(a, a, acc[r][0]);
                acc[r][1] = fma2(b, b, acc[r][1]);
            }
        }
        const ulonglong2 hh = *reinterpret_cast<const ulonglong2 *>(h + j);
        const u64 s = pack2(-k2, -k2);
#pragma unroll
        for (int r = 0; r < RW; ++r) {
            const ulonglong2 t = {fma2(s, acc[r][0], hh.x), fma2(s, acc[r][1], hh.y)};
            *reinterpret_cast<ulonglong2 *>(w + (size_t)r * mp + j) = t;
        }
    }
}
template <int RW, bool DOTS>
__global__ void __launch_bounds__(WARPS * 32, DOTS ? 2 : 3) draw_warps_kernel(const __grid_constant__ Draw P)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowScratch sc[WARPS];
    __shared__ unsigned char bytes[DOTS ? WARPS : 1][ROW_TILE];
    const int mp = P.mp, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const WarpShape<RW, DOTS> shape(mp, P.d);
    float *h = reinterpret_cast<float *>(smem), *w = reinterpret_cast<float *>(smem + (size_t)mp * 4 + (size_t)warp * shape.warp);
    RowRoom M;
    M.list = w + RW * mp;
    M.where = reinterpret_cast<unsigned short *>(M.list + list_room(mp) + ROW_TILE);
    M.tiles = reinterpret_cast<double *>(M.where + list_room(mp) + 2 * ROW_TILE);
    u64 *xs = reinterpret_cast<u64 *>(M.tiles + (mp / ROW_TILE + 1) / 2 * 2);
    M.step = 2 * RW;
    M.bytes = bytes[DOTS ? warp : 0];
    const RowGroup G = {lane, 32, 0, &sc[warp]}, all = {(int)threadIdx.x, WARPS * 32, 0, &sc[0]};
    int turn = 0;
    // units of RW rows, the block's a range of all lanes'
    const unsigned per_lane = (P.rows + RW - 1) / RW;
    const unsigned long long total = (unsigned long long)P.lanes * per_lane;
    const unsigned first = (unsigned)(total * blockIdx.x / gridDim.x), last = (unsigned)(total * (blockIdx.x + 1) / gridDim.x);
    LaneState S;
    unsigned at = first;
#pragma unroll 1
    while (at < last) {
        const unsigned wl = at / per_lane, lane_end = (wl + 1) * per_lane, end = last < lane_end ? last : lane_end;
        enter_lane<WARPS * 32, DOTS>(P, S, P.lane0 + (int)wl, h, all);
        const float *yt = P.yt + (size_t)S.lane * P.d * mp;
#pragma unroll 1
        for (unsigned u = at + warp; u < end; u += WARPS) {
            const int r0 = (int)(u - wl * per_lane) * RW, rows = min(RW, P.rows - r0);
            const size_t row0 = (size_t)S.lane * P.n + P.row0 + r0;
            if (!S.some) {
#pragma unroll 1
                for (int r = 0; r < rows; ++r) draw_none(P, row0 + r, lane, 32);
                continue;
            }
            if (!DOTS) {
                for (int q = lane; q < RW * P.d; q += 32) {
                    const int r = q / P.d, k = q % P.d;
                    const float v = r < rows ? -raw_value(P.x, P.x4, P.dtype, row0 + r, P.d, k) : 0.f;
                    xs[k * RW + r] = pack2(v, v);
                }
                __syncwarp();
                form_warp<RW>(yt, h, xs, w, mp, P.d, S.k2);
                __syncwarp();
            }
#pragma unroll 1
            for (int r = 0; r < rows; ++r) {
                M.w = w + (size_t)r * mp;
                M.x = reinterpret_cast<float *>(xs) + (DOTS ? 0 : 2 * r);
                do_row<DOTS, DOTS>(P, S, row0 + r, G, turn, M, h, DOTS ? P.dots + ((size_t)wl * P.rows + r0 + r) * P.ldo : nullptr);
            }
        }
        at = end;
    }
}

// Longer rows, R to a block: the block's 512 threads form them, then 512 / R threads have a row each.
template <int R, bool DOTS>
struct GroupShape {
    int x;
    size_t all;
    __host__ __device__ GroupShape(int mp, int d)
    {
        x = DOTS ? R * dots_xd(d) * 4 : R * d * 8;
        all = (size_t)mp * 4 + (size_t)R * (mp * 4 + list_room(mp) * 6 + 2 * ROW_TILE * 4 + (mp / ROW_TILE + 1) / 2 * 16) + x;
    }
};
template <int R>
__device__ __forceinline__ void form_rows(const float *yt, const float *h, const u64 *xs, float *w, int mp, int d, float k2)
{
#pragma unroll 1
    for (int j = 4 * threadIdx.x; j < mp; j += 4 * 512) {
        u64 acc[R][2];
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r][0] = acc[r][1] = 0ull;
#pragma unroll 4
        for (int k = 0; k < d; ++k) {
            const ulonglong2 y = *reinterpret_cast<const ulonglong2 *>(yt + (size_t)k * mp + j);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const u64 x = xs[k * R + r], a = add2(y.x, x), b = add2(y.y, x);
                acc[r][0] = fma2(a, a, acc[r][0]);
                acc[r][1] = fma2(b, b, acc[r][1]);
            }
        }
        const ulonglong2 hh = *reinterpret_cast<const ulonglong2 *>(h + j);
        const u64 s = pack2(-k2, -k2);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const ulonglong2 t = {fma2(s, acc[r][0], hh.x), fma2(s, acc[r][1], hh.y)};
            *reinterpret_cast<ulonglong2 *>(w + (size_t)r * mp + j) = t;
        }
    }
}
template <int R, bool DOTS>
__global__ void __launch_bounds__(512, 1) draw_groups_kernel(const __grid_constant__ Draw P)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowScratch sc[R];
    __shared__ unsigned char bytes[DOTS ? 16 : 1][ROW_TILE];
    constexpr int NG = 512 / R;                                  // threads of a row's group
    const int mp = P.mp, tid = threadIdx.x, g = tid / NG, room = list_room(mp), nt2 = (mp / ROW_TILE + 1) / 2 * 2;
    float *h = reinterpret_cast<float *>(smem), *w = h + mp;
    const int lists = room * 3 / 2 + 2 * ROW_TILE;               // floats: weights, and columns of half the size
    u64 *xs = reinterpret_cast<u64 *>(w + (size_t)R * (mp + lists) + (size_t)R * nt2 * 2);
    RowRoom M;
    M.w = w + (size_t)g * mp;
    M.list = w + (size_t)R * mp + (size_t)g * lists;
    M.where = reinterpret_cast<unsigned short *>(M.list + room + ROW_TILE);
    M.tiles = reinterpret_cast<double *>(w + (size_t)R * (mp + lists)) + (size_t)g * nt2;
    M.x = reinterpret_cast<float *>(xs) + (DOTS ? g * dots_xd(P.d) : 2 * g);
    M.step = 2 * R;
    M.bytes = bytes[DOTS ? tid >> 5 : 0];
    const RowGroup G = {tid % NG, NG, 1 + g, &sc[g]}, all = {tid, 512, 0, &sc[0]};
    int turn = 0;
    const unsigned per_lane = (P.rows + R - 1) / R;
    const unsigned long long total = (unsigned long long)P.lanes * per_lane;
    const unsigned first = (unsigned)(total * blockIdx.x / gridDim.x), last = (unsigned)(total * (blockIdx.x + 1) / gridDim.x);
    LaneState S;
    S.lane = -1;
#pragma unroll 1
    for (unsigned t = first; t < last; ++t) {
        const unsigned wl = t / per_lane;
        const int r0 = (int)(t - wl * per_lane) * R, rows = min(R, P.rows - r0);
        if (P.lane0 + (int)wl != S.lane) enter_lane<512, DOTS>(P, S, P.lane0 + (int)wl, h, all);
        const size_t row0 = (size_t)S.lane * P.n + P.row0 + r0;
        if (!S.some) {
#pragma unroll 1
            for (int r = 0; r < rows; ++r) draw_none(P, row0 + r, tid, 512);
            continue;
        }
        if (!DOTS) {
            for (int q = tid; q < R * P.d; q += 512) {
                const int r = q / P.d, k = q % P.d;
                const float v = r < rows ? -raw_value(P.x, P.x4, P.dtype, row0 + r, P.d, k) : 0.f;
                xs[k * R + r] = pack2(v, v);
            }
            __syncthreads();
            form_rows<R>(P.yt + (size_t)S.lane * P.d * mp, h, xs, w, mp, P.d, S.k2);
            __syncthreads();
        }
        if (g < rows) do_row<DOTS, false>(P, S, row0 + g, G, turn, M, h, DOTS ? P.dots + ((size_t)wl * P.rows + r0 + g) * P.ldo : nullptr);
        if (!DOTS) __syncthreads();
    }
}

// Rows of products that are formed again, four warps to a row: among rows that are done in 10 us those that take a
// warp 70 more would be what a launch waits for.
constexpr int LATER_THREADS = 128;
size_t later_smem(int mp, int d) { return GroupShape<1, true>(mp, d).all; }
__global__ void __launch_bounds__(LATER_THREADS, 4) draw_later_kernel(const __grid_constant__ Draw P)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowScratch sc;
    __shared__ unsigned char bytes[LATER_THREADS / 32][ROW_TILE];
    const int mp = P.mp, tid = threadIdx.x, room = list_room(mp), lists = room * 3 / 2 + 2 * ROW_TILE, nt2 = (mp / ROW_TILE + 1) / 2 * 2;
    float *h = reinterpret_cast<float *>(smem);
    RowRoom M;
    M.w = h + mp;
    M.list = M.w + mp;
    M.where = reinterpret_cast<unsigned short *>(M.list + room + ROW_TILE);
    M.tiles = reinterpret_cast<double *>(M.list + lists);
    M.x = reinterpret_cast<float *>(M.tiles + nt2);
    M.step = 0;
    M.bytes = bytes[tid >> 5];
    const RowGroup G = {tid, LATER_THREADS, 0, &sc};
    int turn = 0;
    LaneState S;
    S.lane = -1;
    const unsigned rows = *P.later_n;
#pragma unroll 1
    for (unsigned t = blockIdx.x; t < rows; t += gridDim.x) {
        const long long row = P.later[t];
        const int w = (int)(row / P.n), i = (int)(row % P.n);
        if (w != S.lane) enter_lane<LATER_THREADS, true>(P, S, w, h, G);
        do_row<true, false>(P, S, (size_t)row, G, turn, M, h, P.dots + ((size_t)(w - P.lane0) * P.rows + (i - P.row0)) * P.ldo);
    }
}

size_t exact_smem(const Draw &P) { return (size_t)P.mp / ROW_TILE * 8 + (size_t)dots_xd(P.d) * 8; }

// How a problem is run: the kernel and its rows to a warp or a block, where the exponents come from, and the rows whose
// products are held at a time.
struct Plan {
    int warp_rows, block_rows;                              // one of them; neither: too long for shared memory
    bool dots;
    int lanes, rows, fit;                                   // fit: blocks to an SM
    size_t smem;
    bool fp32() const { return warp_rows || block_rows; }
};
constexpr size_t DRAW_SMEM = 216 * 1024;                    // dynamic; a block has up to 9 KB more, an SM 227 KB
template <int RW, bool DOTS>
bool warps_fit(Plan &p, int mp, int d, size_t most)
{
    p.smem = WarpShape<RW, DOTS>(mp, d).all;
    if (p.smem > most) return false;
    p.warp_rows = RW;
    p.fit = (int)std::min<size_t>(DOTS ? 2 : 3, 226 * 1024 / (p.smem + 10 * 1024));
    return true;
}
template <int R, bool DOTS>
bool groups_fit(Plan &p, int mp, int d)
{
    p.smem = GroupShape<R, DOTS>(mp, d).all;
    if (p.smem > DRAW_SMEM) return false;
    p.block_rows = R;
    p.fit = 1;
    return true;
}
Plan plan_of(const Draw &P)
{
    Plan p = {};
    // Deep clouds whose rows TMA can take.  Below 64 dimensions the products are a small part of a pair's work.
    p.dots = P.dtype == SKB_F32 ? false : P.d >= 64 && (P.dtype != SKB_BF16 || P.d % 8 == 0);
    // A row to a warp while two blocks share an SM, three where that leaves more rows to a warp; then a row to four warps,
    // then to a block.
    const size_t three = 65 * 1024, two = 103 * 1024;
    if (p.dots) (void)(warps_fit<1, true>(p, P.mp, P.d, two) || groups_fit<4, true>(p, P.mp, P.d) || groups_fit<1, true>(p, P.mp, P.d));
    else {
        // (several rows to a warp only where every warp that the GPU holds still has two such units: 8 lanes of 64 rows of 64,
        // 16 us with four rows to a warp, 6 with one)
        const long long rows = (long long)P.W * P.n, warps = 2LL * 3 * WARPS * DRAW_BLOCKS;
        (void)((rows >= 4 * warps && warps_fit<4, false>(p, P.mp, P.d, three)) || (rows >= 2 * warps && warps_fit<2, false>(p, P.mp, P.d, three)) ||
               warps_fit<1, false>(p, P.mp, P.d, two) || groups_fit<4, false>(p, P.mp, P.d) || groups_fit<1, false>(p, P.mp, P.d));
    }
    p.lanes = P.W; p.rows = P.n;
    if (!p.fp32()) p.dots = false;
    if (p.dots) {
        const size_t lane = (size_t)P.n * P.mp * 4;
        if (lane <= DRAW_DOTS_BYTES) p.lanes = (int)std::min<size_t>(P.W, DRAW_DOTS_BYTES / lane);
        else { p.lanes = 1; p.rows = (int)std::max<size_t>(128, DRAW_DOTS_BYTES / ((size_t)P.mp * 4) / 128 * 128); }
        p.rows = std::min(p.rows, P.n);
    }
    return p;
}

// Where the parts of the workspace are; returns its size.
size_t carve(Draw &P, const Plan &p, char *base)
{
    size_t at = 0;
    auto take = [&](size_t bytes) { char *q = base ? base + at : nullptr; at += (bytes + 255) / 256 * 256; return q; };
    P.hn = (double *)take((size_t)P.W * P.mp * 8);
    if (p.dots) {
        P.yn = (float2 *)take((size_t)P.W * P.mp * 8);
        P.xn = (float2 *)take((size_t)P.W * P.n * 8);
        P.dots = (const float *)take((size_t)p.lanes * p.rows * P.mp * 4);
    } else P.yt = (float *)take((size_t)P.W * P.d * P.mp * 4);
    if (p.dots && p.warp_rows) {
        P.launches = ((P.W + p.lanes - 1) / p.lanes) * ((P.n + p.rows - 1) / p.rows);
        P.later_n = (unsigned *)take((size_t)P.launches * 4);
        P.later = (long long *)take((size_t)p.lanes * p.rows * 8);
    }
    P.scratch = (double *)take((size_t)DRAW_EXACT_BLOCKS * P.mp * 8);
    if (p.fp32()) P.list = (long long *)take(((size_t)P.W * P.n + 1) * 8);
    return at;
}

// (limits for any shape: another host thread may set one between this and the launch)
template <int RW, bool DOTS>
void launch_warps(const Draw &P, const Plan &p, cudaStream_t st)
{
    cudaFuncSetAttribute(draw_warps_kernel<RW, DOTS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)DRAW_SMEM / 2);
    const long long units = (long long)P.lanes * ((P.rows + RW - 1) / RW), blocks = (units + WARPS - 1) / WARPS, most = DRAW_BLOCKS * p.fit;
    draw_warps_kernel<RW, DOTS><<<(unsigned)(blocks < most ? blocks : most), WARPS * 32, p.smem, st>>>(P);
}
template <int R, bool DOTS>
void launch_groups(const Draw &P, const Plan &p, cudaStream_t st)
{
    cudaFuncSetAttribute(draw_groups_kernel<R, DOTS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)DRAW_SMEM);
    const long long units = (long long)P.lanes * ((P.rows + R - 1) / R);
    draw_groups_kernel<R, DOTS><<<(unsigned)(units < DRAW_BLOCKS ? units : DRAW_BLOCKS), 512, p.smem, st>>>(P);
}
void launch_draw(const Draw &P, const Plan &p, cudaStream_t st)
{
    if (p.dots) {
        if (p.warp_rows) launch_warps<1, true>(P, p, st);
        else if (p.block_rows == 4) launch_groups<4, true>(P, p, st);
        else launch_groups<1, true>(P, p, st);
    } else if (p.warp_rows == 4) launch_warps<4, false>(P, p, st);
    else if (p.warp_rows == 2) launch_warps<2, false>(P, p, st);
    else if (p.warp_rows == 1) launch_warps<1, false>(P, p, st);
    else if (p.block_rows == 4) launch_groups<4, false>(P, p, st);
    else launch_groups<1, false>(P, p, st);
}

const char *refused(const skb_draw_config *c)
{
    if (c->W < 1 || c->n < 1 || c->m < 1 || c->d < 1) return "W, n, m, d must be >= 1";
    if (c->draws < 1) return "draws must be >= 1";
    if (c->d > 1024) return "d must be at most 1024";
    if (c->n > 262143 || c->m > 262143) return "at most 262143 points per lane";
    if (c->W > 65535) return "at most 65535 lanes";
    if (c->xy_dtype < SKB_F32 || c->xy_dtype > SKB_NV4) return "bad xy_dtype";
    return nullptr;
}

Draw problem(const skb_draw_config *c)
{
    Draw P = {};
    P.dtype = c->xy_dtype; P.W = c->W; P.n = c->n; P.m = c->m; P.d = c->d; P.S = c->draws;
    P.mp = (c->m + ROW_TILE - 1) / ROW_TILE * ROW_TILE;
    P.far = std::min(DRAW_FAR, DRAW_FAR_SUMS / (float)(c->d + 6));
    P.temperature = c->temperature; P.top_k = c->top_k; P.top_p = c->top_p; P.min_p = c->min_p;
    return P;
}

}  // namespace
}  // namespace skb

using namespace skb;

extern "C" size_t sinkhorn_plan_draw_workspace_bytes(const skb_draw_config *cfg)
{
    if (!cfg || refused(cfg)) return 0;
    Draw P = problem(cfg);
    return carve(P, plan_of(P), nullptr);
}

skb_status skb::plan_draw(const void *x, const void *y, const double *g, const float *eps, const float *u, const skb_draw_config *cfg,
                          const int *status, int *index, float *logp)
{
    if (!x || !y || !g || !eps || !u || !cfg || !index) return op_fail(SKB_ERR_NULL, "x, y, g, eps, u, cfg and index are required");
    if (const char *why = refused(cfg)) return op_fail(SKB_ERR_SHAPE, why);
    const size_t need = sinkhorn_plan_draw_workspace_bytes(cfg);
    if (!cfg->workspace || (uintptr_t)cfg->workspace % 256 || cfg->workspace_bytes < need)
        return op_fail(SKB_ERR_WORKSPACE, "workspace missing, not 256-byte aligned or smaller than " + std::to_string(need) + " bytes");
    const bool packed = cfg->xy_dtype == SKB_MX4 || cfg->xy_dtype == SKB_NV4;
    if ((uintptr_t)x % (packed ? 256 : 16) || (uintptr_t)y % (packed ? 256 : 16))
        return op_fail(SKB_ERR_VALUE, "x and y must be 16-byte aligned, 4-bit clouds 256-byte aligned");
    Draw P = problem(cfg);
    P.x = x; P.y = y; P.g = g; P.eps = eps; P.u = u; P.status = status; P.index = index; P.logp = logp;
    if (packed) {
        P.x4 = cloud4_view(x, (size_t)P.W * P.n, P.d, P.dtype);
        P.y4 = cloud4_view(y, (size_t)P.W * P.m, P.d, P.dtype);
    }
    const Plan p = plan_of(P);
    carve(P, p, (char *)cfg->workspace);
    cudaStream_t st = (cudaStream_t)cfg->stream;
    if (!p.dots) transpose_kernel<<<dim3(P.mp / 32, P.W), 256, 0, st>>>(P);
    auto exact = [&] {
        const long long rows = (long long)P.W * P.n;
        draw_exact_kernel<<<(unsigned)(rows < DRAW_EXACT_BLOCKS ? rows : DRAW_EXACT_BLOCKS), 512, exact_smem(P), st>>>(P);
        return op_launched("plan_draw");
    };
    if (!p.fp32()) return exact();
    if (!p.dots) {
        // (a launch counts its rows in 32 bits; 64 cost draws of 256 x 512 rows of 512 56 us of 688)
        const int most = INT_MAX / P.n;
        P.rows = P.n;
        for (P.lane0 = 0; P.lane0 < P.W; P.lane0 += most) {
            P.lanes = std::min(most, P.W - P.lane0);
            launch_draw(P, p, st);
        }
        return exact();
    }
    const dim3 points((P.mp + P.n + 7) / 8, P.W);
    if (P.dtype == SKB_BF16) norms_kernel<true><<<points, 256, 0, st>>>(P);
    else norms_kernel<false><<<points, 256, 0, st>>>(P);
    P.ldo = P.mp;
    for (P.lane0 = 0; P.lane0 < P.W; P.lane0 += p.lanes)
        for (P.row0 = 0; P.row0 < P.n; P.row0 += p.rows) {
            P.lanes = std::min(p.lanes, P.W - P.lane0);
            P.rows = std::min(p.rows, P.n - P.row0);
            const skb_status s = launch_dots(dots_cloud(P.x, P.x4, P.dtype, P.d, (size_t)P.lane0 * P.n + P.row0),
                                             dots_cloud(P.y, P.y4, P.dtype, P.d, (size_t)P.lane0 * P.m), P.dtype, P.lanes, P.rows, P.m,
                                             const_cast<float *>(P.dots), P.ldo, st);
            if (s != SKB_OK) return s;
            launch_draw(P, p, st);
            if (p.warp_rows) {
                cudaFuncSetAttribute(draw_later_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)DRAW_SMEM / 2);
                draw_later_kernel<<<std::min(P.lanes * P.rows, DRAW_BLOCKS * 4), LATER_THREADS, later_smem(P.mp, P.d), st>>>(P);
                ++P.later_n;
            }
        }
    return exact();
}

extern "C" skb_status sinkhorn_plan_draw(const void *x, const void *y, const double *g, const float *eps, const float *u,
                                         const skb_draw_config *cfg, int *index, float *logp)
{
    return plan_draw(x, y, g, eps, u, cfg, nullptr, index, logp);
}
