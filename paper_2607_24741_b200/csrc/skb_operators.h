// What the operators beside the solver (clouds in 4 and 8 bits, their products, maps over them, draws from a coupling, the loss of scores
// against its rows) share on the host.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <string>

#include "../../include/sinkhorn_batch.h"
#include "skb_cloud4.cuh"

namespace skb {

skb_status op_fail(skb_status st, const std::string &msg);     // sets the calling thread's text
skb_status op_launched(const char *what);                       // the launch's status; clears the text where it went well
const char *cloud4_refused(int W, int npts, int d, int format);   // null, or why there is no such cloud
const char *cloud8_refused(int W, int npts, int d);
// Points of a cloud from `row` on, as products take them: bf16 values, or codes, scales and powers of two.
struct DotsCloud {
    const void *data;
    const uint8_t *scales;
    const float *points;
    int row_bytes, sb;
};
DotsCloud dots_cloud(const void *base, const Cloud4 &c, int dtype, int d, size_t row);
// x_i . y_j of W lanes of n and m points (bf16: d a multiple of 8, rows 16-byte aligned), rows of ldo >= m floats.  A lane has
// n rows, or n_out >= n of m_out >= m columns, those past the points zero.
// bf16: sums of DOTS_BF16_PART dimensions by the matrix unit, added in fp32.
constexpr int DOTS_BF16_PART = 64;
skb_status launch_dots(const DotsCloud &x, const DotsCloud &y, int dtype, int W, int n, int m, float *out, long long ldo, cudaStream_t st,
                       int n_out = 0, int m_out = 0);
// The tensor map of W lanes of npts points of row_bytes (a multiple of 16, 16-byte aligned): boxes of 128 bytes of box_points points, 128-byte swizzle.
bool points_map(CUtensorMap *tm, const void *codes, int row_bytes, int npts, int W, int box_points);
// ... and of rows of 128 bytes that lie as shared memory is to have them: boxes of 64 rows.
bool staged_map(CUtensorMap *tm, const void *base, size_t rows);
// ... and of bf16 points (d a multiple of 8, 16-byte aligned): boxes of 64 dimensions of 128 points, 128-byte swizzle.
bool queries_map(CUtensorMap *tm, const void *x, int d, int n, int W);
constexpr int MAP_MAX_SMS = 160;                                // multiprocessors that a map's workspace is sized for
// sinkhorn_plan_draw; lanes whose `status` (null: none) is SKB_LANE_NONFINITE give no draws.
skb_status plan_draw(const void *x, const void *y, const double *g, const float *eps, const float *u, const skb_draw_config *cfg,
                     const int *status, int *index, float *logp);

}  // namespace skb
