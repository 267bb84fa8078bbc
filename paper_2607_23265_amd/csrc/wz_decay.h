// Shared by the kernels of linear attention with a decay for each head
// (wz_decay_attention).
#pragma once

#include "wz_serve.h"

namespace wz {

// log2 of head h's decay, cut to [-200, 0]: its powers are 1 at 0 and zeros in
// fp32 from the lower end on, and a power of zero tokens stays 1.  A NaN stays.
__device__ __forceinline__ float log2_decay(const DecayArgs& p, int h) {
  const float r = p.log_decay[h] * 1.44269504088896341f;
  return r > 0.f ? 0.f : r < -200.f ? -200.f : r;
}

}  // namespace wz
