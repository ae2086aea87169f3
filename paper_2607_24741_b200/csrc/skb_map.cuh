// Images under the entropic map of a stored cloud: what its kernels share.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/sinkhorn_batch.h"
#include "skb_cloud8.cuh"

namespace skb {

constexpr int MAP_TILES_MAX_D = 512;          // queries' depth up to which they stay in shared memory as tiles
constexpr int MAP_TILES_SMEM = 232448;        // shared memory that a block may have

struct Map {
    const uint16_t *x;                        // [W, n, d] bf16
    Cloud8 y, v;                              // bank and its values (the same where there are none of their own)
    const double *g;                          // [W, m], null: zeros
    const float *eps;                         // [W]
    const int *lengths;                       // [W], null: m
    uint16_t *out;                            // [W, n, dv] bf16
    float *lse;                               // [W, n], null: not wanted
    float *part_ml, *part_out;                // splits > 1: [W, n, splits] pairs, [W, n, splits, dv]
    int W, n, m, d, dv, splits;
    int own_values;                           // v is not y
    unsigned char *staged_y, *staged_v;       // many queries: bank and values as bf16 (the same where v is y)
    float *terms;                             // ... and what targets add to exponents, [W, tiles, 128]
    float *sums;                              // ... and blocks' images of what is behind them, where parts are long; null: they are not
};

// Many queries (skb_map_tc.cu): d <= MAP_TILES_MAX_D, P.splits parts of a lane's bank, room for the bank in bf16 and blocks' sums (256-byte aligned).
size_t map_staged_bytes(int W, int n, int m, int d, int dv, bool own_values, int splits);
skb_status launch_map_tiles(Map &P, void *room, int sms, cudaStream_t st);

__device__ __forceinline__ int map_length(const Map &P, int w) { return P.lengths ? min(max(P.lengths[w], 0), P.m) : P.m; }
// log2(e) / eps; NaN, and so are the lane's images, where eps is not a positive number
__device__ __forceinline__ double map_scale(const Map &P, int w)
{
    const float eps = P.eps[w];
    return eps > 0.f && eps <= 3.402823466e38f ? 1.4426950408889634 / (double)eps : __longlong_as_double(0x7ff8000000000000LL);
}
// What a target adds to the exponent of every query, in powers of two; minus infinity: it is masked, whatever its codes.  (What is below fp32's range is
// its lowest value: a finite potential masks nothing by itself.)
__device__ __forceinline__ float map_term(double k, double g, float norm)
{
    const float term = (float)(k * (g - (double)norm));
    return g == -INFINITY ? -INFINITY : term == -INFINITY && norm < INFINITY ? -3.402823466e38f : term;
}
// natural logarithm of the sum of exponentials, from the largest exponent and the sum against it (powers of two) and |x|^2
__device__ __forceinline__ float map_lse(float top, float sum, double k, double xx)
{
    if (sum == 0.f) return -INFINITY;
    return (float)(0.6931471805599453 * ((double)top + (double)log2f(sum) - k * xx));
}

}  // namespace skb
