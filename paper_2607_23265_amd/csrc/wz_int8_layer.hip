// Products of 8-bit integers with an activation and a residual in their
// epilogue, and the two of a gated block (wz_matmul_int_epilogue, wz_gated_int).
#include "wz_int8_tile.h"

namespace wz {

hipError_t launch_matmul_epilogue(const MatmulArgs& p, int out_dtype, hipStream_t s) {
  if (p.M == 0) return hipSuccess;
  return out_dtype == WZ_BF16 ? matmul<uint16_t, kRich>(p, s) : matmul<float, kRich>(p, s);
}

hipError_t launch_gated(const MatmulArgs& p, int out_dtype, hipStream_t s) {
  if (p.M == 0) return hipSuccess;
  return out_dtype == WZ_BF16 ? matmul<uint16_t, kGated>(p, s) : matmul<float, kGated>(p, s);
}

}  // namespace wz
