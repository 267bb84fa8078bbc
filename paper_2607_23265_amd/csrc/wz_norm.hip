// Rows of a residual stream to 8-bit integers behind their root-mean-square
// norm (wz_norm_quantize).
#include "wz_serve.h"

namespace wz {
namespace {

// Eight elements of a row in fp32, from memory and back.
__device__ __forceinline__ void load8(const uint16_t* p, float (&f)[8]) {
  const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = e % 2 ? bf16_hi(v[e / 2]) : bf16_lo(v[e / 2]);
}
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[i + e] = v[e];
  }
}
// f is left as what memory holds then.
__device__ __forceinline__ void store8(uint16_t* p, float (&f)[8]) {
  u32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t lo = f32_to_bf16_rne(f[2 * e]), hi = f32_to_bf16_rne(f[2 * e + 1]);
    v[e] = lo | hi << 16, f[2 * e] = bf16_lo(v[e]), f[2 * e + 1] = bf16_hi(v[e]);
  }
  *reinterpret_cast<u32x4*>(p) = v;
}
__device__ __forceinline__ void store8(float* p, float (&f)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
}

// LANES threads a row (a wave: four rows a workgroup; or the workgroup).  Up to
// CHUNKS chunks of 8 elements a thread stay in registers between the row's sums
// and the rounding (as t = h * weight: the norm's factor is one number a row and
// cancels in the codes); a longer row's others are read again.  Bound by memory:
// 9459 x 3584 in bf16 with a residual, 237 MB, in 41 to 48 us, 5.8 to 4.9 TB/s (the first
// with its result in the last-level cache); 64 rows 4.1 us, a launch and three waits.
template <typename T, int LANES, int CHUNKS>
__global__ __launch_bounds__(256) void k_norm(NormArgs p) {
  __shared__ float red[3][4];
  const int row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, t = threadIdx.x % LANES;
  if (LANES == kWave && row >= p.rows) return;
  const int chunks = p.cols / 8;
  const T* const x = static_cast<const T*>(p.x) + row * p.x_stride;
  const T* const r = p.residual ? static_cast<const T*>(p.residual) + row * p.residual_stride : nullptr;
  T* const total = r ? static_cast<T*>(p.total) + row * p.total_stride : nullptr;
  const T* const stream = r ? total : x;  // what h is read from again
  uint32_t amax = 0;  // of |t| as bits: a NaN is above an infinity, an infinity above every number
  float sum = 0.f;
  auto take = [&](int c, float (&h)[8]) {  // h becomes t
    float w[8];
    load8(p.weight + 8 * c, w);
    if (r) {
      float y[8];
      load8(r + 8 * c, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] += y[e];
      store8(total + 8 * c, h);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum = fmaf(h[e], h[e], sum);
      h[e] *= w[e];
      amax = max(amax, __float_as_uint(h[e]) & 0x7fffffffu);
    }
  };
  float kept[CHUNKS][8];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
    if (t + i * LANES < chunks) load8(x + 8 * (t + i * LANES), kept[i]);
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
    if (t + i * LANES < chunks) take(t + i * LANES, kept[i]);
  for (int c = t + CHUNKS * LANES; c < chunks; c += LANES) {
    float h[8];
    load8(x + 8 * c, h);
    take(c, h);
  }
  auto wave_sum = [](float v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
  };
#pragma unroll
  for (int o = 32; o; o >>= 1) amax = max(amax, uint32_t(__shfl_xor(int(amax), o, kWave)));
  sum = wave_sum(sum);
  auto row_sum = [&](int i, float v) {  // of the row's waves, in their order
    if constexpr (LANES > kWave) {
      if (__lane_id() == 0) red[i][threadIdx.x / kWave] = v;
      __syncthreads();
      v = (red[i][0] + red[i][1]) + (red[i][2] + red[i][3]);
    }
    return v;
  };
  if constexpr (LANES > kWave) {
    if (__lane_id() == 0) red[1][threadIdx.x / kWave] = __uint_as_float(amax);
    sum = row_sum(0, sum);
#pragma unroll
    for (int i = 0; i < 4; ++i) amax = max(amax, __float_as_uint(red[1][i]));
  }
  const bool fine = amax < 0x7f800000u;
  float unit = 1.f, eps = p.eps;
  // (the same for all of a row's threads) squares past fp32, or with eps: of h / 2^80, and eps by as much
  if (fine && !(sum + eps < INFINITY)) {
    float again = 0.f;
    for (int c = t; c < chunks; c += LANES) {
      float h[8];
      load8(stream + 8 * c, h);
#pragma unroll
      for (int e = 0; e < 8; ++e) again = fmaf(h[e] * 0x1p-80f, h[e] * 0x1p-80f, again);
    }
    sum = row_sum(2, wave_sum(again)), unit = 0x1p-80f, eps *= 0x1p-80f, eps *= 0x1p-80f;
  }
  const float top = fmaxf(__uint_as_float(amax), 0x1p-100f), up = 127.f / top;
  if (t == 0)
    p.scale[row] = fine ? (top / 127.f) / sqrtf(sum / float(p.cols) + eps) * unit : __uint_as_float(0x7fc00000u);
  auto put = [&](int c, const float (&y)[8]) {
    uint32_t v[2] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e / 4] |= uint32_t(fine ? int(rintf(y[e] * up)) & 0xff : 0) << (8 * (e % 4));
    *reinterpret_cast<u32x2*>(p.q + row * p.q_stride + 8 * c) = u32x2{v[0], v[1]};
  };
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
    if (t + i * LANES < chunks) put(t + i * LANES, kept[i]);
  for (int c = t + CHUNKS * LANES; c < chunks; c += LANES) {
    float h[8], w[8];
    load8(stream + 8 * c, h);
    load8(p.weight + 8 * c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] *= w[e];
    put(c, h);
  }
}

// Measured (us, bf16 with a residual; a wave to a row, a workgroup with 2 chunks a thread,
// with 8): 9459 x 512 9.1, 13.8, 23.2; 9459 x 1024 13.4, 16.6, 25.2; 9459 x 2048 26.5,
// 24.0, 28.8; 9459 x 3584 53.5, 40.7, 53.9; 4096 x 8192 54.6, 46.1, 43.3; 2048 x 16384
// 71.6, 49.4, 39.3.  Of 64 rows the same choices are the fastest but for one: 64 x 1024
// 4.1, 3.5, 3.5.
template <typename T>
hipError_t norm(const NormArgs& p, hipStream_t s) {
  const dim3 block(256);
  if (p.cols <= 1024)
    hipLaunchKernelGGL((k_norm<T, kWave, 2>), dim3((p.rows + 3) / 4), block, 0, s, p);
  else if (p.cols <= 4096)
    hipLaunchKernelGGL((k_norm<T, 256, 2>), dim3(p.rows), block, 0, s, p);
  else
    hipLaunchKernelGGL((k_norm<T, 256, 8>), dim3(p.rows), block, 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs& p, int dtype, hipStream_t s) {
  if (p.rows == 0) return hipSuccess;
  return dtype == WZ_BF16 ? norm<uint16_t>(p, s) : norm<float>(p, s);
}

}  // namespace wz
