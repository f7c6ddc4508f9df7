// The backward pass of an attention plan (dnb_attn_bwd.hip), for dnb_attn.hip.
#pragma once

#include "dnb_attn_dev.h"

namespace dnb {
namespace attn {
// token: with the work of dq split over the keys
hipError_t launch_backward(const Args& A, bool bf16, bool token, hipStream_t st);
// bytes at Args::part that it takes
size_t backward_part_bytes(int64_t rq, int64_t rk, int n, int kv, int per, int d, bool bf16);
}
}  // namespace dnb
