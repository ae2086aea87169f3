// Partners drawn from the rows of a coupling: row i of a lane is the distribution over j with weights
//     w_j = 2^(z_j - max z),  z_j = k (g_j - |x_i - y_j|^2),  k = log2(e) / (eps T),
// cut down by top-k, top-p and min-p (skb_draw_row.cuh), and a draw for each uniform number that is given.  The row's own
// potential drops out.  The plan is not stored: a block forms the weights of a few rows in shared memory, cuts and draws, and
// goes on to the next rows.
//
// The indices are those of the definition in float64.  The weights are formed in fp32, with a bound on their error; a row in
// which some comparison falls inside the bound is decided again by the whole block in float64, first with exact weights
// for the entries above 2^-22 of the largest alone, then, should that not do, for all.
//
// Two ways to the exponents:
//   differences   |x - y|^2 in fp32 from a transposed copy of y, R rows to a block: two operations a dimension and pair,
//                 two columns to an instruction
//   products      deep bf16 and 4-bit clouds: x . y from the tensor cores (skb_dots.cu) for as many rows at a time as stay in
//                 the L2 cache, z = k (g - |y|^2) + 2 k x . y
// Rows of more than DRAW_MAX_M entries do not fit shared memory: they are decided in float64 alone, weights in the workspace.
#include <cuda_runtime.h>
#include <math_constants.h>
#include <limits.h>

#include "skb_cloud4.cuh"
#include "skb_draw_row.cuh"
#include "skb_operators.h"

namespace skb {
namespace {

constexpr int DRAW_MAX_BLOCKS = 444;                 // 148 SMs, three blocks each: rows of scratch in the workspace
constexpr int DRAW_LONG_BLOCKS = 148;
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
    float *yn, *xn;                                  // [W][mp], [W][n] squared norms (products)
    const float *dots;                               // rows row0 .. row0 + rows - 1 of lanes lane0 .. lane0 + lanes - 1
    double *scratch;                                 // [blocks][mp]
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
__device__ __forceinline__ float ex2(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Transposed copy of y and k g, 32 points to a block.  Masked points get coordinates of zero, whatever theirs are.
__global__ void __launch_bounds__(256) transpose_kernel(const Draw P)
{
    __shared__ float tile[32][33];
    __shared__ int masked[32];
    const int w = blockIdx.y, j0 = blockIdx.x * 32, tid = threadIdx.x, col = tid & 31, part = tid >> 5;
    const Lane L = lane_of(P, w);
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

// |point|^2 in float64, by one warp
__device__ __forceinline__ double square_of(const void *base, const Cloud4 &c, int dtype, size_t row, int d)
{
    double s = 0.0;
    for (int k = threadIdx.x & 31; k < d; k += 32) {
        const double v = (double)raw_value(base, c, dtype, row, d, k);
        s = fma(v, v, s);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    return s;
}
// Squared norms of both clouds and k (g - |y|^2), a warp to a point.
__global__ void __launch_bounds__(256) norms_kernel(const Draw P)
{
    const int w = blockIdx.y, i = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (i < P.mp) {
        const double g = i < P.m ? P.g[(size_t)w * P.m + i] : -CUDART_INF;
        const bool masked = g == -CUDART_INF;
        const double s = masked ? 0.0 : square_of(P.y, P.y4, P.dtype, (size_t)w * P.m + i, P.d);
        if (lane == 0) {
            P.hn[(size_t)w * P.mp + i] = masked ? g : lane_of(P, w).k2 * (g - s);
            P.yn[(size_t)w * P.mp + i] = (float)s;
        }
        return;
    }
    const int r = i - P.mp;
    if (r >= P.n) return;
    const double s = square_of(P.x, P.x4, P.dtype, (size_t)w * P.n + r, P.d);
    if (lane == 0) P.xn[(size_t)w * P.n + r] = (float)s;
}

__device__ __forceinline__ void put_draw(const Draw &P, size_t at, int index, float logp)
{
    P.index[at] = index;
    if (P.logp) P.logp[at] = logp;
}

// Draws of one row from weights and their cut, shared out to the group's warps.  True if all of this warp's were sure.
template <typename Real>
__device__ bool draw_all(const Draw &P, size_t row, const Real *w, const RowCut<Real> &cut, const Real *tiles, double delta, int warp, int warps)
{
    const double total = row_total(tiles, P.mp / ROW_TILE);
    bool sure = true;
    for (int s = warp; s < P.S; s += warps) {
        const float u = P.u[row * P.S + s];
        int j = -1;
        double wj = 0.0;
        if (u >= 0.f && u < 1.f) {
            const bool good = row_draw(w, cut, tiles, P.mp / ROW_TILE, total, (double)u, delta, j, wj);
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

// One row in float64 by the whole block.  wf, scale: the row's fp32 weights and a bound on their relative error; null: none.
// xs: the point's coordinates, `step` floats apart.
__device__ __noinline__ void decide_row(const Draw &P, const Lane &L, int w, int i, const float *xs, int step, const float *wf, double error,
                                        double *wd, double *tiles, RowScratch *sc, int *flag)
{
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5;
    const RowGroup G = {tid, nt, 0, sc};
    const size_t row = (size_t)w * P.n + i;
    const double *hn = P.hn + (size_t)w * P.mp;
    for (int tier = wf ? 0 : 1; tier < 2; ++tier) {
        const float floor_ = tier == 0 ? 2.384185791015625e-7f : -1.f;      // 2^-22
        double top = -CUDART_INF;
        int bad = 0;
        if (P.yt) {
            const float *yt = P.yt + (size_t)w * P.d * P.mp;
            for (int j = tid; j < P.mp; j += nt) {
                if (wf && !(wf[j] > floor_)) continue;
                double c = 0.0;
                for (int k = 0; k < P.d; ++k) {
                    const double e = (double)xs[k * step] - (double)yt[(size_t)k * P.mp + j];
                    c = fma(e, e, c);
                }
                const double z = hn[j] == -CUDART_INF ? -CUDART_INF : fma(-L.k2, c, hn[j]);
                wd[j] = z;
                top = fmax(top, z);
                bad |= !(z <= 1.7e308);
            }
        } else {
            for (int j = warp; j < P.mp; j += nt >> 5) {
                if (wf && !(wf[j] > floor_)) continue;
                double z = -CUDART_INF;
                if (hn[j] != -CUDART_INF) {
                    double c = 0.0;
                    for (int k = lane; k < P.d; k += 32) {
                        const double e = (double)xs[k * step] - (double)raw_value(P.y, P.y4, P.dtype, (size_t)w * P.m + j, P.d, k);
                        c = fma(e, e, c);
                    }
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) c += __shfl_xor_sync(0xffffffffu, c, off);
                    z = L.k2 * (P.g[(size_t)w * P.m + j] - c);
                }
                if (lane == 0) wd[j] = z;
                top = fmax(top, z);
                bad |= !(z <= 1.7e308);
            }
        }
        double some = 0.0;
        top = G.largest(top);
        G.add(some, bad);                                           // (a barrier: wd is written)
        if (bad || top == -CUDART_INF) { draw_none(P, row, tid, nt); return; }
        double mass = 0.0, rest = 0.0;
        int count = 0, unused = 0;
        for (int j = tid; j < P.mp; j += nt) {
            double v;
            if (wf && !(wf[j] > floor_)) { v = (double)wf[j]; rest += v; }
            else v = exp2(wd[j] - top);
            wd[j] = v;
            mass += v;
            count += v > 0.0;
        }
        G.add(mass, count);
        G.add(rest, unused);
        const double delta = tier == 0 ? 4.0 * error * rest / mass + 1e-12 : 0.0;
        RowCut<double> cut;
        bool sure = row_cut(wd, P.mp, G, L.cuts, mass, count, delta, cut, tiles);
        if (sure && tier == 0 && cut.lowest < 2.0 * floor_) sure = false;
        if (sure) {
            if (tid == 0) *flag = 0;
            __syncthreads();
            if (!draw_all(P, row, wd, cut, tiles, delta, warp, nt >> 5) && lane == 0) *flag = 1;
            __syncthreads();
            sure = *flag == 0;
        }
        __syncthreads();
        if (sure) return;
    }
}

// Rows too long for shared memory: a block to a row, float64 throughout.
__global__ void __launch_bounds__(512) draw_long_kernel(const Draw P)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowScratch sc;
    __shared__ int flag;
    double *tiles = reinterpret_cast<double *>(smem);
    float *xs = reinterpret_cast<float *>(tiles + P.mp / ROW_TILE);
    for (long long t = blockIdx.x; t < (long long)P.W * P.n; t += gridDim.x) {
        const int w = (int)(t / P.n), i = (int)(t % P.n);
        const Lane L = lane_of(P, w);
        __syncthreads();
        if (!L.ok) { draw_none(P, (size_t)t, threadIdx.x, blockDim.x); continue; }
        for (int k = threadIdx.x; k < P.d; k += blockDim.x) xs[k] = raw_value(P.x, P.x4, P.dtype, (size_t)t, P.d, k);
        __syncthreads();
        decide_row(P, L, w, i, xs, 1, nullptr, 0.0, P.scratch + (size_t)blockIdx.x * P.mp, tiles, &sc, &flag);
    }
}

size_t long_smem(const Draw &P) { return (size_t)P.mp / ROW_TILE * 8 + (size_t)P.d * 4; }

// Where the parts of the workspace are; returns its size.
size_t carve(Draw &P, char *base)
{
    size_t at = 0;
    auto take = [&](size_t bytes) { char *p = base ? base + at : nullptr; at += (bytes + 255) / 256 * 256; return p; };
    P.hn = (double *)take((size_t)P.W * P.mp * 8);
    P.yt = (float *)take((size_t)P.W * P.d * P.mp * 4);
    P.scratch = (double *)take((size_t)DRAW_LONG_BLOCKS * P.mp * 8);
    return at;
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
    return carve(P, nullptr);
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
    carve(P, (char *)cfg->workspace);
    cudaStream_t st = (cudaStream_t)cfg->stream;
    transpose_kernel<<<dim3(P.mp / 32, P.W), 256, 0, st>>>(P);
    const long long rows = (long long)P.W * P.n;
    draw_long_kernel<<<(unsigned)(rows < DRAW_LONG_BLOCKS ? rows : DRAW_LONG_BLOCKS), 512, long_smem(P), st>>>(P);
    return op_launched("plan_draw");
}
