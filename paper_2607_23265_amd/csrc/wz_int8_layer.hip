// Products of 8-bit integers with an activation and a residual in their
// epilogue, and the two of a gated block (wz_matmul_int_epilogue, wz_gated_int).
//
// Measured: 64 x 3584 x 14336 onto a residual in 14.4 us with its weights in the last-level
// cache, 22 with weights from memory (10.2 at a copy's rate), 9459 of these rows in 425 to 451
// (2.2 POP/s, as the library's 8192^3 product); 12544 x 3584 x 1152 with gelu in 81 to 90 (1.2
// POP/s: with so few steps of K a tile's ends and its activations are half of its time).
// Gated: 64 x 14336 x 3584 in 24.2 to 26.3 (3.9 to 4.3 TB/s of weights), 1286 rows in 163 to 172
// (1.6 POP/s: 1286 rows are 10.05 tiles of 128, and the rounds of the CUs are not full), 9459 in
// 859 to 916 (2.2 POP/s).
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
