// The backward pass of an attention plan (dnb_attn_bwd.hip), for dnb_attn.hip.
#pragma once

#include "dnb_attn_dev.h"

namespace dnb {
namespace attn {
hipError_t launch_backward(const Args& A, bool bf16, hipStream_t st);
}
}  // namespace dnb
