// What the operators beside the solver (4-bit clouds, their products, draws from a coupling) share on the host.
#pragma once
#include <cuda_runtime.h>
#include <string>

#include "../../include/sinkhorn_batch.h"

namespace skb {

skb_status op_fail(skb_status st, const std::string &msg);     // sets the calling thread's text
skb_status op_launched(const char *what);                       // the launch's status; clears the text where it went well
const char *cloud4_refused(int W, int npts, int d, int format);   // null, or why there is no such cloud

}  // namespace skb
