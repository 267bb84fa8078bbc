// Rows to 8-bit integers and their product with weights held the same way
// (wz_quantize_rows, wz_matmul_int).
#include "wz_serve.h"

namespace wz {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// One workgroup a row; the row stays in registers between its largest
// magnitude and its rounding, so it is read once.
template <typename In>
__global__ __launch_bounds__(kThreads) void k_quantize(const In* x, int64_t x_stride, int cols, int8_t* q,
                                                       int64_t q_stride, float* scale) {
  constexpr int kMost = 65536 / (8 * kThreads);  // chunks of 8 a thread at the widest row
  __shared__ uint32_t red[4];
  const int row = blockIdx.x, chunks = cols / 8;
  const In* src = x + row * x_stride;
  uint32_t amax = 0;  // largest magnitude as bits: a NaN is above an infinity, an infinity above every number
  for (int i = threadIdx.x; i < chunks; i += kThreads) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t u;
      if constexpr (sizeof(In) == 2) u = uint32_t(src[8 * i + e]) << 16;
      else u = __float_as_uint(src[8 * i + e]);
      amax = max(amax, u & 0x7fffffffu);
    }
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) amax = max(amax, uint32_t(__shfl_xor(int(amax), o, kWave)));
  if (__lane_id() == 0) red[threadIdx.x / kWave] = amax;
  __syncthreads();
  amax = max(max(red[0], red[1]), max(red[2], red[3]));
  const bool fine = amax < 0x7f800000u;
  const float top = fmaxf(__uint_as_float(amax), 0x1p-100f), up = fine ? 127.f / top : 0.f;
  if (threadIdx.x == 0) scale[row] = fine ? top / 127.f : __uint_as_float(0x7fc00000u);
  for (int i = threadIdx.x; i < chunks; i += kThreads) {
    uint32_t y[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float f;
      if constexpr (sizeof(In) == 2) f = __uint_as_float(uint32_t(src[8 * i + e]) << 16);
      else f = src[8 * i + e];
      const int v = fine ? int(rintf(f * up)) : 0;
      const uint32_t byte = uint32_t(v) & 0xffu;
      y[e / 4] = e % 4 ? y[e / 4] | byte << (8 * (e % 4)) : byte;
    }
    *reinterpret_cast<u32x2*>(q + row * q_stride + 8 * i) = u32x2{y[0], y[1]};
  }
}

// 64 x 64 of the product, a wave 32 x 32 of it, straight from memory.
template <typename Out>
__global__ __launch_bounds__(kThreads) void k_matmul(const int8_t* a, int64_t a_stride, const float* a_scale,
                                                     const int8_t* w, int64_t w_stride, const float* w_scale,
                                                     const float* bias, int M, int N, int K, Out* out,
                                                     int64_t out_stride) {
  const int lane = __lane_id(), wave = threadIdx.x / kWave, c = lane & 15, g = lane >> 4;
  const int m0 = blockIdx.y * 64 + 32 * (wave / 2), n0 = blockIdx.x * 64 + 32 * (wave % 2);
  i32x4 acc[2][2] = {};
  for (int k = 0; k < K; k += 64) {
    const int at = k + 16 * g;
    i32x4 x[2], y[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[i] = at < K ? *reinterpret_cast<const i32x4*>(a + int64_t(min(m0 + 16 * i + c, M - 1)) * a_stride + at) : i32x4{};
      y[i] = at < K ? *reinterpret_cast<const i32x4*>(w + int64_t(min(n0 + 16 * i + c, N - 1)) * w_stride + at) : i32x4{};
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[i], y[j], acc[i][j], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = m0 + 16 * i + 4 * g + e, n = n0 + 16 * j + c;
        if (m < M && n < N) {
          float v = float(acc[i][j][e]) * a_scale[m] * w_scale[n];
          if (bias) v += bias[n];
          if constexpr (sizeof(Out) == 2) out[m * out_stride + n] = f32_to_bf16_rne(v);
          else out[m * out_stride + n] = v;
        }
      }
}

}  // namespace

hipError_t launch_quantize(const void* x, int64_t x_stride, int rows, int cols, int in_dtype, int8_t* q,
                           int64_t q_stride, float* scale, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  if (in_dtype == WZ_BF16)
    hipLaunchKernelGGL((k_quantize<uint16_t>), dim3(rows), dim3(kThreads), 0, s, static_cast<const uint16_t*>(x), x_stride, cols, q, q_stride, scale);
  else
    hipLaunchKernelGGL((k_quantize<float>), dim3(rows), dim3(kThreads), 0, s, static_cast<const float*>(x), x_stride, cols, q, q_stride, scale);
  return hipGetLastError();
}

hipError_t launch_matmul(const MatmulArgs& p, int out_dtype, hipStream_t s) {
  if (p.M == 0) return hipSuccess;
  const dim3 grid((p.N + 63) / 64, (p.M + 63) / 64), block(kThreads);
  if (out_dtype == WZ_BF16)
    hipLaunchKernelGGL((k_matmul<uint16_t>), grid, block, 0, s, p.a, p.a_stride, p.a_scale, p.w, p.w_stride, p.w_scale, p.bias, p.M, p.N, p.K, static_cast<uint16_t*>(p.out), p.out_stride);
  else
    hipLaunchKernelGGL((k_matmul<float>), grid, block, 0, s, p.a, p.a_stride, p.a_scale, p.w, p.w_stride, p.w_scale, p.bias, p.M, p.N, p.K, static_cast<float*>(p.out), p.out_stride);
  return hipGetLastError();
}

}  // namespace wz
