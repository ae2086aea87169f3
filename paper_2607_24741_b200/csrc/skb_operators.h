// What the operators beside the solver (4-bit clouds, their products, draws from a coupling) share on the host.
#pragma once
#include <cuda_runtime.h>
#include <string>

#include "../../include/sinkhorn_batch.h"

namespace skb {

skb_status op_fail(skb_status st, const std::string &msg);     // sets the calling thread's text
skb_status op_launched(const char *what);                       // the launch's status; clears the text where it went well
const char *cloud4_refused(int W, int npts, int d, int format);   // null, or why there is no such cloud
// x_i . y_j of clouds of type `dtype` (bf16: d a multiple of 8, both 16-byte aligned), n rows of ldo >= m floats to a lane
skb_status launch_dots(int dtype, const void *x, const void *y, int W, int n, int m, int d, float *out, long long ldo, cudaStream_t st);

}  // namespace skb
