// Partners drawn from the rows of a coupling: row i of a lane is the distribution over j with weights
//     w_j = 2^(z_j - max z),  z_j = k (g_j - |x_i - y_j|^2),  k = log2(e) / (eps T),
// cut down by top-k, top-p and min-p (skb_draw_row.cuh), and a draw for each uniform number that is given.  The row's own
// potential drops out.  The plan is not stored: a block forms the weights of a few rows in shared memory, cuts and draws, and
// goes on to the next rows.
//
// The indices are those of the definition in float64.  The weights are formed in fp32, with bounds on their errors, cut and drawn
// from (skb_draw_quick.cuh).  A row in which some comparison falls inside the bounds is formed again, to fp32's last place,
// where it weighs more than 2^-22 of its largest entry, and decided again with sums in double (skb_draw_row.cuh); what that
// leaves open goes on a list, for a kernel that decides in float64 throughout.
//
// Two ways to the exponents:
//   differences   |x - y|^2 in fp32 from a transposed copy of y, R rows to a block: two operations a dimension and pair,
//                 two columns to an instruction
//   products      deep bf16 and 4-bit clouds: x . y from the tensor cores (skb_dots.cu) for as many rows at a time as stay in
//                 the L2 cache, z = k (g - |y|^2) + 2 k x . y
// Rows that do not fit shared memory (from some 49 000 entries on) are decided in float64 alone, weights in the workspace.
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
constexpr size_t DRAW_DOTS_BYTES = (size_t)64 << 20; // products that are held at a time: half of the L2 cache

struct Draw {
    const void *x, *y;
    Cloud4 x4, y4;
    const double *g;
    const float *eps, *temperature, *top_p, *min_p, *u;
    const int *top_k;
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
__device__ __forceinline__ float raw_value(const void *base, const Cloud4 &c, int dtype, size_t row, int d, int k)
{
    if (dtype == SKB_F32) return ((const float *)base)[row * d + k];
    if (dtype == SKB_BF16) return __uint_as_float((uint32_t)((const uint16_t *)base)[row * d + k] << 16);
    return cloud4_value(c, row, k);
}
// Transposed copy of y and k g, 32 points to a block.  Masked points get coordinates of zero, whatever theirs are.
__global__ void __launch_bounds__(256) transpose_kernel(const Draw P)
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
        if (j < P.mp) P.hn[(size_t)w * P.mp + j] = g == -CUDART_INF ? g : L.k2 * g;
    }
    __syncthreads();
    float *yt = P.yt + (size_t)w * P.d * P.mp;
    if (P.d <= 8) {
        if (part < P.d) yt[(size_t)part * P.mp + j0 + col] = masked[col] ? 0.f : raw_value(P.y, P.y4, P.dtype, (size_t)w * P.m + j0 + col, P.d, part);
        return;
    }
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

// Eight dimensions of point `row` from k on, k a multiple of 8; zeros past the last (k < the padded depth).
__device__ __forceinline__ void eight_values(const void *data, const Cloud4 &c, int dtype, size_t row, int d, int k, float (&v)[8])
{
    if (dtype == SKB_BF16) {
        const uint4 a = *reinterpret_cast<const uint4 *>((const uint16_t *)data + row * d + k);
        const uint32_t b[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(b[i] << 16); v[2 * i + 1] = __uint_as_float(b[i] & 0xffff0000u); }
    } else {
        const uint32_t b = *reinterpret_cast<const uint32_t *>(c.codes + row * c.cb + k / 2);
        const float s = cloud4_scale(c, row, k);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = e2m1_value(b >> (4 * i)) * s;
    }
}
__host__ __device__ inline int dots_xd(int d) { return (d + 31) / 32 * 32; }
// |point|^2 in float64, by one warp; prefix: the mean of the squared norms of its first 16, 32, ... dimensions.
__device__ __forceinline__ double square_of(const void *base, const Cloud4 &c, int dtype, size_t row, int d, double &prefix)
{
    double s = 0.0;
    float p = 0.f;
    const int steps = (d + 15) / 16, chunks = dtype == SKB_BF16 ? d / 8 : dots_xd(d) / 8;
    for (int q = threadIdx.x & 31; q < chunks; q += 32) {
        float v[8], f = 0.f;
        eight_values(base, c, dtype, row, d, 8 * q, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = v[i] * v[i];                             // exact: at most 16 bits
            s += (double)a;
            f += a;
        }
        p = fmaf(f, (float)max(steps - q / 2, 1), p);
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
__global__ void __launch_bounds__(256) norms_kernel(const Draw P)
{
    const int w = blockIdx.y, i = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    double p = 0.0;
    if (blockIdx.x == 0 && w == 0 && threadIdx.x == 0) P.list[0] = 0;
    if (i < P.mp) {
        const double g = i < P.m ? P.g[(size_t)w * P.m + i] : -CUDART_INF;
        const bool masked = g == -CUDART_INF;
        const double s = masked ? 0.0 : square_of(P.y, P.y4, P.dtype, (size_t)w * P.m + i, P.d, p);
        if (lane == 0) {
            P.hn[(size_t)w * P.mp + i] = masked ? g : lane_of(P, w).k2 * (g - s);
            P.yn[(size_t)w * P.mp + i] = make_float2((float)s, (float)p);
        }
        return;
    }
    const int r = i - P.mp;
    if (r >= P.n) return;
    const double s = square_of(P.x, P.x4, P.dtype, (size_t)w * P.n + r, P.d, p);
    if (lane == 0) P.xn[(size_t)w * P.n + r] = make_float2((float)s, (float)p);
}

__device__ __forceinline__ void put_draw(const Draw &P, size_t at, int index, float logp)
{
    P.index[at] = index;
    if (P.logp) P.logp[at] = logp;
}

// Draws of one row from weights and their cut, shared out to the group's warps.  True if all of this warp's were sure.
template <typename Real>
__device__ bool draw_all(const Draw &P, size_t row, const Real *w, const RowCut<Real> &cut, const double *tiles, const RowError &err, int warp, int warps)
{
    const double total = row_total(tiles, P.mp / ROW_TILE);
    bool sure = true;
    for (int s = warp; s < P.S; s += warps) {
        const float u = P.u[row * P.S + s];
        int j = -1;
        double wj = 0.0;
        if (u >= 0.f && u < 1.f) {
            const bool good = row_draw(w, cut, tiles, P.mp / ROW_TILE, total, (double)u, err, j, wj);
            if (!good) { sure = false; continue; }
        }
        if ((threadIdx.x & 31) == 0) put_draw(P, row * P.S + s, j, j < 0 ? CUDART_NAN_F : (float)log(wj / total));
    }
    return sure;
}
__device__ void draw_none(const Draw &P, size_t row, int t, int nt)
{
    for (int s = t; s < P.S; s += nt) put_draw(P, row * P.S + s, -1, CUDART_NAN_F);
}


// Rows in float64, a block to a row: those of the list, or all (rows too long for shared memory).
__global__ void __launch_bounds__(512) draw_exact_kernel(const Draw P)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowScratch sc;
    double *tiles = reinterpret_cast<double *>(smem), *xs = tiles + P.mp / ROW_TILE, *wd = P.scratch + (size_t)blockIdx.x * P.mp;
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5, xd = dots_xd(P.d);
    const RowGroup G = {tid, nt, 0, &sc};
    const long long rows = P.list ? P.list[0] : (long long)P.W * P.n;
    for (long long t = blockIdx.x; t < rows; t += gridDim.x) {
        const long long row = P.list ? P.list[1 + t] : t;
        const int w = (int)(row / P.n);
        const Lane L = lane_of(P, w);
        const double *hn = P.hn + (size_t)w * P.mp;
        __syncthreads();
        if (!L.ok) { draw_none(P, (size_t)row, tid, nt); continue; }
        for (int k = tid; k < xd; k += nt) xs[k] = k < P.d ? (double)raw_value(P.x, P.x4, P.dtype, (size_t)row, P.d, k) : 0.0;
        __syncthreads();
        double top = -CUDART_INF;
        int bad = 0;
        if (P.yt) {
            const float *yt = P.yt + (size_t)w * P.d * P.mp;
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
            // eight threads to a point, four points to a warp
            const int part = lane & 7, chunks = P.dtype == SKB_BF16 ? P.d / 8 : xd / 8;
            for (int j0 = 4 * warp; j0 < P.mp; j0 += 4 * (nt >> 5)) {
                const int j = j0 + (lane >> 3);
                const bool is = hn[j] != -CUDART_INF;
                double c = 0.0;
                if (is) {
#pragma unroll 4
                    for (int q = part; q < chunks; q += 8) {
                        float y[8];
                        eight_values(P.y, P.y4, P.dtype, (size_t)w * P.m + j, P.d, 8 * q, y);
#pragma unroll
                        for (int i = 0; i < 8; ++i) { const double e = xs[8 * q + i] - (double)y[i]; c = fma(e, e, c); }
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
        double mass = 0.0;
        int count = 0;
        top = G.largest(top);
        G.add(mass, bad);                                           // (a barrier: wd is written)
        if (bad || top == -CUDART_INF) { draw_none(P, (size_t)row, tid, nt); continue; }
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
        draw_all(P, (size_t)row, wd, cut, tiles, none, warp, nt >> 5);
        __syncthreads();
    }
}

// R rows of a lane at a time, NT threads: weights in shared memory by all threads, then a group of NT / R threads to a row.
//   tiles [R][mp / 128], w [R][mp], lists [R][mp / 4], h [mp]: the lane's hn less its largest, as fp32; xs: -x, twice each, [d][R] pairs
//   (differences), or x [R][xd] of rows that are formed again (products)
// Error of an exponent t = log2 w at a depth q below the row's largest, A = |largest t|:
//   differences  h <= 0 and the scaled distance h - t are at most A + q; d + 2 roundings of the distance, three of the
//                scale and t, one of h: (d + 6) (A + q) 2^-24
//   products     2 k |x . y| is at most B = 2 k |x| max |y|, and after each 16 dimensions at most the same of those
//                prefixes, on average no more than B' (from the root mean squares of the prefixes' norms).  The matrix unit
//                cuts off where it adds products to a sum: a unit in the last place of the sum, at most 2^-23 of it, for each 16, and
//                two more: (d / 16) B' 2^-23 + 2 B 2^-23; the roundings of h, scale and t: (3 B + 3 (A + q)) 2^-24
// The exponential adds 2^-22 and 2^-24 q of the difference that it is taken of, the additions of weights 2^-24 each.
template <int R, int NT>
struct DrawShape {
    static size_t smem(int mp, int d, bool dots)
    {
        return (size_t)R * (mp / ROW_TILE * 8 + (size_t)mp * 5) + (size_t)mp * 4 + (dots ? (size_t)R * dots_xd(d) * 4 : (size_t)R * d * 8);
    }
};

// Exponents of the block's rows from coordinate differences, RPT rows and four columns to a thread.
template <int R, int NT, int RPT>
__device__ __forceinline__ void form_rows(const float *yt, const float *h, const u64 *xs, float *w, int mp, int d, float k2)
{
    constexpr int RG = R / RPT, CT = NT / RG;
    const int ct = threadIdx.x % CT, r0 = threadIdx.x / CT * RPT;
    const float ninf = -k2;
    for (int j = 4 * ct; j < mp; j += 4 * CT) {
        u64 acc[RPT][2];
#pragma unroll
        for (int r = 0; r < RPT; ++r) acc[r][0] = acc[r][1] = 0ull;
#pragma unroll 2
        for (int k = 0; k < d; ++k) {
            const ulonglong2 y = *reinterpret_cast<const ulonglong2 *>(yt + (size_t)k * mp + j);
#pragma unroll
            for (int r = 0; r < RPT; r += 2) {
                ulonglong2 x = {0ull, 0ull};
                if constexpr (RPT >= 2) x = *reinterpret_cast<const ulonglong2 *>(xs + k * R + r0 + r);
                else x.x = xs[k * R + r0];
#pragma unroll
                for (int q = 0; q < (RPT >= 2 ? 2 : 1); ++q) {
                    const u64 a = add2(y.x, q ? x.y : x.x), b = add2(y.y, q ? x.y : x.x);
                    acc[r + q][0] = fma2(a, a, acc[r + q][0]);
                    acc[r + q][1] = fma2(b, b, acc[r + q][1]);
                }
            }
        }
        const ulonglong2 hh = *reinterpret_cast<const ulonglong2 *>(h + j);
        const u64 s = pack2(ninf, ninf);
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
            const ulonglong2 t = {fma2(s, acc[r][0], hh.x), fma2(s, acc[r][1], hh.y)};
            *reinterpret_cast<ulonglong2 *>(w + (size_t)(r0 + r) * mp + j) = t;
        }
    }
}

// Mass, number and largest of a row's weights, and the mass of those at most ROW_FLOOR.
struct RowSums {
    double mass, rest;
    int count;
    float top;
};
__device__ __forceinline__ RowSums sum_row(const RowGroup &G, const float *w, int mp)
{
    RowSums r = {0.0, 0.0, 0, 0.f};
    for (int j = 4 * G.t; j < mp; j += 4 * G.nt) {
        float v[4];
        load4(w + j, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r.mass += (double)v[i];
            r.rest += v[i] > ROW_FLOOR ? 0.0 : (double)v[i];
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
    for (int q = warp; q < P.mp / ROW_TILE; q += warps) {
        const int j = q * ROW_TILE + 4 * lane;
        float v[4];
        load4(w + j, v);
        if (!(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])) > ROW_FLOOR)) continue;
        double c[4] = {0.0, 0.0, 0.0, 0.0};
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
__device__ __forceinline__ void refine_products(const Draw &P, double k2, int wl, const double *hn, const float *x, float magic, double base,
                                                float *w, unsigned char *list, int warp, int warps)
{
    const int lane = threadIdx.x & 31, part = lane & 7, col = lane >> 3;
    const int chunks = P.dtype == SKB_BF16 ? P.d / 8 : dots_xd(P.d) / 8;
    for (int q = warp; q < P.mp / ROW_TILE; q += warps) {
        float v[4];
        load4(w + q * ROW_TILE + 4 * lane, v);
        int n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned ball = __ballot_sync(0xffffffffu, v[i] > ROW_FLOOR);
            if (v[i] > ROW_FLOOR) list[n + __popc(ball & ((1u << lane) - 1u))] = (unsigned char)(4 * lane + i);
            n += __popc(ball);
        }
        __syncwarp();
        for (int e0 = 0; e0 < n; e0 += 4) {
            const int j = q * ROW_TILE + list[min(e0 + col, n - 1)];
            const size_t row = (size_t)wl * P.m + j;
            const u64 m2 = pack2(magic, magic);
            u64 sum = m2, low = 0ull;
#pragma unroll 4
            for (int c = part; c < chunks; c += 8) {
                float y[8];
                eight_values(P.y, P.y4, P.dtype, row, P.d, 8 * c, y);
                const ulonglong2 xa = reinterpret_cast<const ulonglong2 *>(x + 8 * c)[0], xb = reinterpret_cast<const ulonglong2 *>(x + 8 * c)[1];
                const u64 xv[4] = {xa.x, xa.y, xb.x, xb.y};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u64 yv = pack2(y[2 * i], y[2 * i + 1]), t = fma2(xv[i], yv, sum);
                    low = add2(low, fma2(xv[i], yv, sub2(sum, t)));
                    sum = t;
                }
            }
            float a, b, la, lb;
            unpack2(sub2(sum, m2), a, b);                            // exact
            unpack2(low, la, lb);
            double dot = ((double)a + (double)b) + ((double)la + (double)lb);
#pragma unroll
            for (int off = 1; off < 8; off *= 2) dot += __shfl_xor_sync(0xffffffffu, dot, off);
            if (part == 0 && e0 + col < n) w[j] = (float)exp2(fma(2.0 * k2, dot, hn[j]) - base);
        }
        __syncwarp();
    }
}

// Sums of two floats and a count over the group, added in one order.
__device__ __forceinline__ void group_sums(const RowGroup &G, float &a, float &b, unsigned &n, int &turn)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, off);
        b += __shfl_xor_sync(0xffffffffu, b, off);
    }
    n = __reduce_add_sync(0xffffffffu, n);
    if (G.nt == 32) return;
    turn ^= 1;
    if ((G.t & 31) == 0) {
        unsigned *p = G.sc->part[turn][G.t >> 5];
        p[0] = __float_as_uint(a); p[1] = __float_as_uint(b); p[2] = n;
    }
    G.sync();
    a = b = 0.f;
    n = 0;
    for (int q = 0; q < G.nt >> 5; ++q) {
        const unsigned *p = G.sc->part[turn][q];
        a += __uint_as_float(p[0]); b += __uint_as_float(p[1]); n += p[2];
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
    for (int q = 0; q < G.nt >> 5; ++q) v = v && G.sc->part[turn][q][0] != 0;
    return v;
}

// A row once more: what weighs more than ROW_FLOOR to fp32's last place, what does not is `off` of itself off.  x: -x, `step`
// apart (differences), or room for a row (products), whose bound is `bound`.
template <bool DOTS>
__device__ __noinline__ bool again(const Draw &P, const Lane &L, int wl, size_t row, const RowGroup &G, double base, float off, float bound, float *x,
                                   int step, float *w, double *tiles, unsigned char *list)
{
    const double *hn = P.hn + (size_t)wl * P.mp;
    if (DOTS) {
        const int xd = dots_xd(P.d);
        for (int k = G.t; k < xd; k += G.nt) x[k] = k < P.d ? raw_value(P.x, P.x4, P.dtype, row, P.d, k) : 0.f;
        // twice to four times the bound, and half as much again: sums within the bound stay in its binade
        const float magic = 1.5f * __uint_as_float((__float_as_uint(bound * 4.f) & 0x7f800000u) + 0x00800000u);
        G.sync();
        refine_products(P, L.k2, wl, hn, x, magic, base, w, list, G.t >> 5, G.nt >> 5);
    } else refine_differences(P, L.k2, hn, P.yt + (size_t)wl * P.d * P.mp, x, step, base, w, G.t >> 5, G.nt >> 5);
    G.sync();
    const RowSums sums = sum_row(G, w, P.mp);
    if (!(sums.mass <= 3e38)) return false;
    const RowError fine = {2.0 * (5.9604645e-8 * sums.mass + sums.rest * off), 2.f * 5.9604645e-8f, 0.f};
    RowCut<float> cut;
    if (!row_cut(w, P.mp, G, L.cuts, sums.top, sums.mass, sums.count, fine, cut, tiles) || cut.lowest < 2.f * ROW_FLOOR) return false;
    return draw_all(P, row, w, cut, tiles, fine, G.t >> 5, G.nt >> 5);
}

template <int R, int NT, bool DOTS>
__global__ void __launch_bounds__(NT, NT > 256 ? 1 : 3) draw_kernel(const Draw P)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowScratch sc[R];
    __shared__ unsigned char lists[DOTS ? NT / 32 : 1][ROW_TILE];
    constexpr int NG = NT / R;                                   // threads of a row's group
    const int mp = P.mp, ntiles = mp / ROW_TILE, tid = threadIdx.x, lane = tid & 31, xd = dots_xd(P.d);
    double *tiles_all = reinterpret_cast<double *>(smem);
    float *w_all = reinterpret_cast<float *>(tiles_all + (R * ntiles + 1) / 2 * 2);
    float *h = w_all + (size_t)R * (mp + mp / 4);
    u64 *xs = reinterpret_cast<u64 *>(h + mp);
    float *x1 = reinterpret_cast<float *>(xs);
    const int g = tid / NG;
    const RowGroup G = {tid % NG, NG, 1 + g, &sc[g]}, all = {tid, NT, 0, &sc[0]};
    float *w = w_all + (size_t)g * mp;
    double *tiles = tiles_all + (size_t)g * ntiles;
    unsigned *units = reinterpret_cast<unsigned *>(tiles);       // (never at the same time)
    constexpr float u24 = 5.9604645e-8f;

    const int per_lane = (P.rows + R - 1) / R;
    const long long total = (long long)P.lanes * per_lane, first = total * blockIdx.x / gridDim.x, last = total * (blockIdx.x + 1) / gridDim.x;
    int at_lane = -1, turn = 0;
    float y_max = 0.f, y_prefix = 0.f;
    double h_top = 0.0;
    bool some = false;
    for (long long t = first; t < last; ++t) {
        const int wl = (int)(t / per_lane), r0 = (int)(t % per_lane) * R, lanew = P.lane0 + wl, i0 = P.row0 + r0;
        const int rows = min(R, P.rows - r0);
        const size_t row0 = (size_t)lanew * P.n + i0;
        const Lane L = lane_of(P, lanew);
        const double *hn = P.hn + (size_t)lanew * mp;
        if (!L.ok) {
            for (int r = 0; r < rows; ++r) draw_none(P, row0 + r, tid, NT);
            continue;
        }
        if (lanew != at_lane) {
            // the lane's largest k g_j (- |y_j|^2), and the others less that
            __syncthreads();
            double top = -CUDART_INF;
            float far = 0.f, prefix = 0.f;
            for (int j = tid; j < mp; j += NT) {
                top = fmax(top, hn[j]);
                if (DOTS) {
                    const float2 s = P.yn[(size_t)lanew * mp + j];
                    far = fmaxf(far, s.x);
                    prefix = fmaxf(prefix, s.y);
                }
            }
            h_top = all.largest(top);
            if (DOTS) { y_max = sqrtf(all.largest(far)); y_prefix = sqrtf(all.largest(prefix)); }
            some = h_top != -CUDART_INF;
            for (int j = tid; j < mp; j += NT) h[j] = some ? (float)(hn[j] - h_top) : 0.f;
            at_lane = lanew;
            __syncthreads();
        }
        if (!some) {
            for (int r = 0; r < rows; ++r) draw_none(P, row0 + r, tid, NT);
            continue;
        }
        const float k2 = (float)L.k2;
        const float *yt = P.yt + (size_t)lanew * P.d * mp;
        if (!DOTS) {
            for (int q = tid; q < R * P.d; q += NT) {
                const int r = q / P.d, k = q % P.d;
                const float v = r < rows ? -raw_value(P.x, P.x4, P.dtype, row0 + r, P.d, k) : 0.f;
                xs[k * R + r] = pack2(v, v);
            }
            __syncthreads();
            // rows too short for all threads to have four columns of them: fewer rows to a thread
            if constexpr (R == 8) {
                if (mp > 512) form_rows<R, NT, 8>(yt, h, xs, w_all, mp, P.d, k2);
                else if (mp > 256) form_rows<R, NT, 4>(yt, h, xs, w_all, mp, P.d, k2);
                else if (mp > 128) form_rows<R, NT, 2>(yt, h, xs, w_all, mp, P.d, k2);
                else form_rows<R, NT, 1>(yt, h, xs, w_all, mp, P.d, k2);
            } else form_rows<R, NT, R>(yt, h, xs, w_all, mp, P.d, k2);
            __syncthreads();
        }
        if (g < rows) {
            const size_t row = row0 + g;
            float top = -CUDART_INF_F;
            if (DOTS) {
                const float *dots = P.dots + ((size_t)wl * P.rows + r0 + g) * P.ldo;
                const float two_k = (float)(2.0 * L.k2);
#pragma unroll 8
                for (int j = 4 * G.t; j < mp; j += 4 * NG) {
                    float v[4], hh[4];
                    load4(dots + j, v);
                    load4(h + j, hh);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[i] = hh[i] == -CUDART_INF_F ? -CUDART_INF_F : fmaf(two_k, v[i], hh[i]);
                        top = fmaxf(top, v[i]);
                    }
                    *reinterpret_cast<float4 *>(w + j) = make_float4(v[0], v[1], v[2], v[3]);
                }
            } else {
#pragma unroll 4
                for (int j = 4 * G.t; j < mp; j += 4 * NG) {
                    float v[4];
                    load4(w + j, v);
                    top = fmaxf(fmaxf(top, fmaxf(v[0], v[1])), fmaxf(v[2], v[3]));
                }
            }
            top = group_largest(G, top, turn);
            // nothing left in fp32's range, a NaN or an infinite exponent: float64 tells which
            bool sure = false;
            if (top != -CUDART_INF_F) {
                float mass = 0.f, depth = 0.f;
                unsigned count = 0;
#pragma unroll 4
                for (int j = 4 * G.t; j < mp; j += 4 * NG) {        // (each thread's own: no barrier yet)
                    float v[4];
                    load4(w + j, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float below = top - v[i];
                        v[i] = ex2_fast(-below);
                        count += v[i] > 0.f;
                        depth += v[i] > 0.f ? v[i] * below : 0.f;
                    }
                    *reinterpret_cast<float4 *>(w + j) = make_float4(v[0], v[1], v[2], v[3]);
                    mass += (v[0] + v[1]) + (v[2] + v[3]);
                }
                const unsigned own = count;
                group_sums(G, mass, depth, count, turn);
                G.sync();
                if (mass <= 3e38f) {
                    const float A = fabsf(top), adds = u24 * (float)(12 + mp / (4 * NG));
                    float fixed, slope, x_norm = 0.f;               // of an exponent: fixed + slope q
                    if (DOTS) {
                        const float2 xn = P.xn[row];
                        x_norm = sqrtf(xn.x);
                        const float b = 2.f * k2 * x_norm * y_max, bp = 2.f * k2 * sqrtf(xn.y) * y_prefix;
                        slope = 3.f * u24;
                        fixed = u24 * (2.f * (float)((P.d + 15) / 16) * bp + 7.f * b + 3.f * A);
                    } else {
                        slope = (float)(P.d + 6) * u24;
                        fixed = slope * A;
                    }
                    fixed = 0.6932f * fixed + 2.4e-7f;
                    slope = 0.6932f * (slope + u24);
                    // (of two weights: twice the error of one)
                    const RowError err = {1.0, 2.f * fixed, 2.f * slope};
                    const float off = fixed + 24.f * slope;
                    if (off < 0.01f) {
                        const float unit = QUICK_ONE / mass;
                        // (roundings to units: half of one for each thread of a pass, and for each of 32 in a tile, twice)
                        const QuickSlack slack = {1.02f * fixed * QUICK_ONE, (2.f * adds + slope * depth / mass) * QUICK_ONE + (float)(NG + 32 * ntiles)};
                        QuickCut cut;
                        sure = quick_cut(w, mp, G, L.cuts, count, own, unit, slack, err, w_all + (size_t)R * mp + (size_t)g * (mp / 4), mp / 4, cut, turn);
                        if (sure) {
                            quick_tiles(w, ntiles, G, cut.tau, unit, units);
                            G.sync();
                            const unsigned whole = quick_total(units, ntiles);
                            for (int s = G.t >> 5; s < P.S; s += NG >> 5) {
                                const float u = P.u[row * P.S + s];
                                int j = -1;
                                float wj = 0.f;
                                if (u >= 0.f && u < 1.f && !quick_draw(w, ntiles, cut.tau, unit, units, whole, u, slack, j, wj)) { sure = false; continue; }
                                if (lane == 0) put_draw(P, row * P.S + s, j, j < 0 ? CUDART_NAN_F : logf(wj * unit / (float)whole));
                            }
                        }
                        sure = group_all(G, sure, turn);
                        if (!sure) {
                            // once more, with better weights for what counts
                            G.sync();
                            sure = again<DOTS>(P, L, lanew, row, G, h_top + (double)top, off, x_norm * y_max, DOTS ? x1 + (size_t)g * xd : x1 + 2 * g,
                                               2 * R, w, tiles, lists[DOTS ? tid >> 5 : 0]);
                            sure = group_all(G, sure, turn);
                        }
                    }
                }
            }
            if (!sure && G.t == 0) P.list[1 + (long long)atomicAdd((unsigned long long *)P.list, 1ull)] = (long long)row;
            G.sync();
        }
        if (!DOTS) __syncthreads();
    }
}

size_t exact_smem(const Draw &P) { return (size_t)P.mp / ROW_TILE * 8 + (size_t)dots_xd(P.d) * 8; }

// How a problem is run: rows to a block, where the exponents come from, and the rows whose products are held at a time.
struct Plan {
    int R;                                                  // 8, 4, 1; 0: too long for shared memory
    bool dots;
    int lanes, rows;
    size_t smem;
};
constexpr size_t DRAW_SMEM = 216 * 1024;                     // dynamic; a block has 8 KB more, an SM 227 KB
Plan plan_of(const Draw &P)
{
    Plan p = {};
    // Deep clouds whose rows TMA can take.  Below 64 dimensions the products are a small part of a pair's work.
    p.dots = P.dtype == SKB_F32 ? false : P.d >= 64 && (P.dtype != SKB_BF16 || P.d % 8 == 0);
    const size_t s8 = DrawShape<8, 256>::smem(P.mp, P.d, p.dots), s4 = DrawShape<4, 512>::smem(P.mp, P.d, p.dots),
                 s1 = DrawShape<1, 512>::smem(P.mp, P.d, p.dots);
    // eight rows while two blocks share an SM, four while one fits
    if (s8 + 10 * 1024 <= DRAW_SMEM / 2) { p.R = 8; p.smem = s8; }
    else if (s4 + 64 <= DRAW_SMEM) { p.R = 4; p.smem = s4; }
    else if (s1 + 64 <= DRAW_SMEM) { p.R = 1; p.smem = s1; }
    p.smem += 64;
    p.lanes = P.W; p.rows = P.n;
    if (p.dots && p.R) {
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
    if (p.dots && p.R) {
        P.yn = (float2 *)take((size_t)P.W * P.mp * 8);
        P.xn = (float2 *)take((size_t)P.W * P.n * 8);
        P.dots = (const float *)take((size_t)p.lanes * p.rows * P.mp * 4);
    } else P.yt = (float *)take((size_t)P.W * P.d * P.mp * 4);
    P.scratch = (double *)take((size_t)DRAW_EXACT_BLOCKS * P.mp * 8);
    if (p.R) P.list = (long long *)take(((size_t)P.W * P.n + 1) * 8);
    return at;
}

template <int R, int NT, bool DOTS>
void launch_draw(const Draw &P, const Plan &p, cudaStream_t st)
{
    // (the limit for any shape: another host thread may set it between this and the launch)
    cudaFuncSetAttribute(draw_kernel<R, NT, DOTS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(R == 8 ? DRAW_SMEM / 2 : DRAW_SMEM));
    const long long tiles = (long long)P.lanes * ((P.rows + R - 1) / R);
    const size_t fit = NT > 256 ? 1 : std::min<size_t>(3, 226 * 1024 / (p.smem + 10 * 1024));
    const long long most = (long long)(DRAW_BLOCKS * fit);
    draw_kernel<R, NT, DOTS><<<(unsigned)(tiles < most ? tiles : most), NT, p.smem, st>>>(P);
}
template <bool DOTS>
void launch_draw(const Draw &P, const Plan &p, cudaStream_t st)
{
    if (p.R == 8) launch_draw<8, 256, DOTS>(P, p, st);
    else if (p.R == 4) launch_draw<4, 512, DOTS>(P, p, st);
    else launch_draw<1, 512, DOTS>(P, p, st);
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

extern "C" skb_status sinkhorn_plan_draw(const void *x, const void *y, const double *g, const float *eps, const float *u,
                                         const skb_draw_config *cfg, int *index, float *logp)
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
    P.x = x; P.y = y; P.g = g; P.eps = eps; P.u = u; P.index = index; P.logp = logp;
    if (packed) {
        P.x4 = cloud4_view(x, (size_t)P.W * P.n, P.d, P.dtype);
        P.y4 = cloud4_view(y, (size_t)P.W * P.m, P.d, P.dtype);
    }
    const Plan p = plan_of(P);
    carve(P, p, (char *)cfg->workspace);
    cudaStream_t st = (cudaStream_t)cfg->stream;
    if (!p.dots || !p.R) transpose_kernel<<<dim3(P.mp / 32, P.W), 256, 0, st>>>(P);
    auto exact_rows = [&] {
        const long long rows = (long long)P.W * P.n;
        draw_exact_kernel<<<(unsigned)(rows < DRAW_EXACT_BLOCKS ? rows : DRAW_EXACT_BLOCKS), 512, exact_smem(P), st>>>(P);
        return op_launched("plan_draw");
    };
    if (!p.R) return exact_rows();
    if (!p.dots) {
        P.lanes = P.W; P.rows = P.n;
        launch_draw<false>(P, p, st);
        return exact_rows();
    }
    norms_kernel<<<dim3((P.mp + P.n + 7) / 8, P.W), 256, 0, st>>>(P);
    P.ldo = P.mp;
    for (P.lane0 = 0; P.lane0 < P.W; P.lane0 += p.lanes)
        for (P.row0 = 0; P.row0 < P.n; P.row0 += p.rows) {
            P.lanes = std::min(p.lanes, P.W - P.lane0);
            P.rows = std::min(p.rows, P.n - P.row0);
            const skb_status s = launch_dots(dots_cloud(P.x, P.x4, P.dtype, P.d, (size_t)P.lane0 * P.n + P.row0),
                                             dots_cloud(P.y, P.y4, P.dtype, P.d, (size_t)P.lane0 * P.m), P.dtype, P.lanes, P.rows, P.m,
                                             const_cast<float *>(P.dots), P.ldo, st);
            if (s != SKB_OK) return s;
            launch_draw<true>(P, p, st);
        }
    return exact_rows();
}
