// Rows to 8-bit integers and their product with weights held the same way
// (wz_quantize_rows, wz_matmul_int).
#include <cmath>

#include "wz_int8_tile.h"

namespace wz {
namespace {

// ---------------------------------------------------------------------------
// Rows to integers
// ---------------------------------------------------------------------------

// LANES threads a row (a wave: four rows a workgroup; or the workgroup); up to
// CHUNKS chunks of 8 elements a thread stay in registers between the row's
// largest magnitude and the rounding, so that the row is read once (twice,
// the second time from L2, where it is longer than that).
template <typename In, int LANES, int CHUNKS>
__global__ __launch_bounds__(256) void k_quantize(const In* x, int64_t x_stride, int rows, int cols, int8_t* q,
                                                  int64_t q_stride, float* scale) {
  constexpr int kWords = sizeof(In) == 2 ? 4 : 8;  // 32-bit words of a chunk
  __shared__ uint32_t red[4];
  const int row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, t = threadIdx.x % LANES;
  const int chunks = cols / 8;
  if (LANES == kWave && row >= rows) return;
  const In* src = x + row * x_stride;
  auto get = [&](int c, uint32_t (&u)[kWords]) {
#pragma unroll
    for (int i = 0; i < kWords; i += 4) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(src + 8 * c + i * (4 / sizeof(In)));
#pragma unroll
      for (int e = 0; e < 4; ++e) u[i + e] = v[e];
    }
  };
  auto element = [](const uint32_t (&u)[kWords], int e) {
    if constexpr (sizeof(In) == 2) return e % 2 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16;
    else return u[e];
  };
  // the largest magnitude as bits: a NaN is above an infinity, an infinity above every number
  uint32_t amax = 0, kept[CHUNKS][kWords];
  auto take = [&](const uint32_t (&u)[kWords]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = max(amax, element(u, e) & 0x7fffffffu);
  };
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
    if (t + i * LANES < chunks) get(t + i * LANES, kept[i]);
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
    if (t + i * LANES < chunks) take(kept[i]);
  for (int c = t + CHUNKS * LANES; c < chunks; c += LANES) {
    uint32_t u[kWords];
    get(c, u);
    take(u);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) amax = max(amax, uint32_t(__shfl_xor(int(amax), o, kWave)));
  if constexpr (LANES > kWave) {
    if (__lane_id() == 0) red[threadIdx.x / kWave] = amax;
    __syncthreads();
    amax = max(max(red[0], red[1]), max(red[2], red[3]));
  }
  const bool fine = amax < 0x7f800000u;
  const float top = fmaxf(__uint_as_float(amax), 0x1p-100f), up = 127.f / top;
  if (t == 0) scale[row] = fine ? top / 127.f : __uint_as_float(0x7fc00000u);
  auto put = [&](int c, const uint32_t (&u)[kWords]) {
    uint32_t y[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int v = fine ? int(rintf(__uint_as_float(element(u, e)) * up)) : 0;
      y[e / 4] = e % 4 ? y[e / 4] | (uint32_t(v) & 0xffu) << (8 * (e % 4)) : uint32_t(v) & 0xffu;
    }
    *reinterpret_cast<u32x2*>(q + row * q_stride + 8 * c) = u32x2{y[0], y[1]};
  };
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
    if (t + i * LANES < chunks) put(t + i * LANES, kept[i]);
  for (int c = t + CHUNKS * LANES; c < chunks; c += LANES) {
    uint32_t u[kWords];
    get(c, u);
    put(c, u);
  }
}

template <typename In>
hipError_t quantize(const In* x, int64_t x_stride, int rows, int cols, int8_t* q, int64_t q_stride, float* scale,
                    hipStream_t s) {
  // A wave to a row, or a workgroup: 9459 rows of 512, 1024, 2048 and 2560 columns
  // of bf16 5.4, 8.6, 13.0 and 16.2 us against 8.9, 10.8, 13.2 and 14.7 (64 rows of
  // 2048 4.3 and 3.5).  Two chunks a thread hold 4096 columns, eight 16 384: 1286
  // rows of 3584 columns 5.1 and 5.4 us, 9459 of 8192 45 and 40.
  const dim3 block(256);
  if (cols <= 2048)
    hipLaunchKernelGGL((k_quantize<In, kWave, 4>), dim3((rows + 3) / 4), block, 0, s, x, x_stride, rows, cols, q,
                       q_stride, scale);
  else if (cols <= 4096)
    hipLaunchKernelGGL((k_quantize<In, 256, 2>), dim3(rows), block, 0, s, x, x_stride, rows, cols, q, q_stride, scale);
  else
    hipLaunchKernelGGL((k_quantize<In, 256, 8>), dim3(rows), block, 0, s, x, x_stride, rows, cols, q, q_stride, scale);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const void* x, int64_t x_stride, int rows, int cols, int in_dtype, int8_t* q,
                           int64_t q_stride, float* scale, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  return in_dtype == WZ_BF16
             ? quantize(static_cast<const uint16_t*>(x), x_stride, rows, cols, q, q_stride, scale, s)
             : quantize(static_cast<const float*>(x), x_stride, rows, cols, q, q_stride, scale, s);
}

hipError_t launch_matmul(const MatmulArgs& p, int out_dtype, hipStream_t s) {
  if (p.M == 0) return hipSuccess;
  return out_dtype == WZ_BF16 ? matmul<uint16_t, kPlain>(p, s) : matmul<float, kPlain>(p, s);
}

}  // namespace wz
