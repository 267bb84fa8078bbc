// Rows to 8-bit integers and their product with weights held the same way
// (wz_quantize_rows, wz_matmul_int).
#include "wz_serve.h"

namespace wz {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

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
  const dim3 block(256);
  if (cols <= 2048)
    hipLaunchKernelGGL((k_quantize<In, kWave, 4>), dim3((rows + 3) / 4), block, 0, s, x, x_stride, rows, cols, q, q_stride, scale);
  else if (cols <= 4096)
    hipLaunchKernelGGL((k_quantize<In, 256, 2>), dim3(rows), block, 0, s, x, x_stride, rows, cols, q, q_stride, scale);
  else
    hipLaunchKernelGGL((k_quantize<In, 256, 8>), dim3(rows), block, 0, s, x, x_stride, rows, cols, q, q_stride, scale);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The product
// ---------------------------------------------------------------------------

// One element of the result, in the order the header states.
template <typename Out>
__device__ __forceinline__ Out finish(int acc, float sa, float sw, float bias) {
  const float v = float(acc) * sa * sw + bias;
  if constexpr (sizeof(Out) == 2) return f32_to_bf16_rne(v);
  else return v;
}

__device__ __align__(16) int g_zeros[4];  // what a lane behind the end of a row reads

// Few rows: the weights are read once and the sum over k is what there is to
// share.  Eight waves of a workgroup take the 64-byte steps of k in turn, for
// 16 MT rows by 16 NT columns, straight from memory into the fragments, and
// add up their integers through LDS.
constexpr int kSkinnyWaves = 8;
template <typename Out, int MT, int NT>
__global__ __launch_bounds__(kSkinnyWaves* kWave) void k_matmul_skinny(MatmulArgs p) {
  constexpr int BM = 16 * MT, BN = 16 * NT, kDepth = 4;
  __shared__ int red[kSkinnyWaves][BM * BN];
  const int lane = __lane_id(), w = threadIdx.x / kWave, c = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * BN, m0 = blockIdx.y * BM;
  const int8_t *ap[MT], *wp[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) ap[i] = p.a + int64_t(min(m0 + 16 * i + c, p.M - 1)) * p.a_stride + 16 * g;
#pragma unroll
  for (int i = 0; i < NT; ++i) wp[i] = p.w + int64_t(min(n0 + 16 * i + c, p.N - 1)) * p.w_stride + 16 * g;
  const int8_t* const zeros = reinterpret_cast<const int8_t*>(g_zeros);
  i32x4 acc[MT][NT] = {};
  const int steps = (p.K + 63) / 64;
  for (int s0 = w; s0 < steps; s0 += kSkinnyWaves * kDepth) {
    i32x4 x[kDepth][MT], y[kDepth][NT];
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      const int at = (s0 + d * kSkinnyWaves) * 64;
      const bool in = at + 16 * g < p.K;
#pragma unroll
      for (int i = 0; i < NT; ++i) y[d][i] = *reinterpret_cast<const i32x4*>(in ? wp[i] + at : zeros);
#pragma unroll
      for (int i = 0; i < MT; ++i) x[d][i] = *reinterpret_cast<const i32x4*>(in ? ap[i] + at : zeros);
    }
#pragma unroll
    for (int d = 0; d < kDepth; ++d)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[d][i], y[d][j], acc[i][j], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) red[w][(16 * i + 4 * g + e) * BN + 16 * j + c] = acc[i][j][e];
  __syncthreads();
  Out* const out = static_cast<Out*>(p.out);
  for (int i = threadIdx.x; i < BM * BN; i += kSkinnyWaves * kWave) {
    const int m = m0 + i / BN, n = n0 + i % BN;
    if (m >= p.M || n >= p.N) continue;
    int sum = 0;
#pragma unroll
    for (int k = 0; k < kSkinnyWaves; ++k) sum += red[k][i];
    out[m * p.out_stride + n] = finish<Out>(sum, p.a_scale[m], p.w_scale[n], p.bias ? p.bias[n] : 0.f);
  }
}

// 16 bytes a lane from a buffer to LDS, lane after lane from `to` on (the
// same in every lane); zeros for an offset behind the buffer's end.
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, int8_t* to, int offset, int uniform) {
  typedef __attribute__((address_space(3))) void* lds_ptr;
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)to, 16, offset, uniform, 0, 0);
}

// Many rows: tiles of BM x BN, WM x WN waves, 128 bytes of k at a time through
// two buffers of LDS that the loads write directly while the other one is
// worked on.  Chunk c of 16 bytes of row r lies at chunk c ^ (r & 7), so that
// eight lanes that read eight rows hit all banks; the loads' lanes fetch in
// that order.
constexpr int kStep = 128;
template <typename Out, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN* kWave) void k_matmul_tile(MatmulArgs p, int tiles_m, int tiles_n) {
  constexpr int kWaves = WM * WN, MT = BM / WM / 32, NT = BN / WN / 32;
  constexpr int kLoadsA = BM / 8 / kWaves, kLoadsB = BN / 8 / kWaves;  // of 8 rows each, a wave
  __shared__ __align__(16) int8_t a0[BM * kStep], b0[BN * kStep], a1[BM * kStep], b1[BN * kStep];
  const int lane = __lane_id(), w = threadIdx.x / kWave, c = lane & 31, g = lane >> 5;

  // Workgroups go to the XCDs in turn: each XCD gets a run of tiles that lie
  // together (columns of 8 row tiles), whose rows and weights its L2 holds.
  const int tiles = tiles_m * tiles_n, per = (tiles + kXcds - 1) / kXcds;
  const int t = (blockIdx.x % kXcds) * per + blockIdx.x / kXcds;
  if (blockIdx.x / kXcds >= per || t >= tiles) return;
  constexpr int kBand = 8;
  const int band = t / (kBand * tiles_n), in_band = t % (kBand * tiles_n);
  const int band_rows = min(kBand, tiles_m - band * kBand);
  const int tm = band * kBand + in_band % band_rows, tn = in_band / band_rows;
  const int m0 = tm * BM, n0 = tn * BN;

  // a row behind the last one is behind its buffer's end and reads as zeros;
  // so is, by its offset, what lies behind the end of a row
  const int lr = lane / 8, lc = 16 * ((lane % 8) ^ lr);  // row of the eight and byte that this lane fetches
  const __amdgpu_buffer_rsrc_t abuf = make_rsrc(p.a + int64_t(m0) * p.a_stride, min(BM, p.M - m0) * int(p.a_stride));
  const __amdgpu_buffer_rsrc_t bbuf = make_rsrc(p.w + int64_t(n0) * p.w_stride, min(BN, p.N - n0) * int(p.w_stride));
  int ao[kLoadsA], bo[kLoadsB];
#pragma unroll
  for (int i = 0; i < kLoadsA; ++i) ao[i] = ((w * kLoadsA + i) * 8 + lr) * int(p.a_stride) + lc;
#pragma unroll
  for (int i = 0; i < kLoadsB; ++i) bo[i] = ((w * kLoadsB + i) * 8 + lr) * int(p.w_stride) + lc;
  auto fetch = [&](int8_t* a, int8_t* b, int k) {
    const bool in = k + lc < p.K;
#pragma unroll
    for (int i = 0; i < kLoadsA; ++i)
      load_to_lds(abuf, a + (w * kLoadsA + i) * 8 * kStep, in ? ao[i] : kOOB, k);
#pragma unroll
    for (int i = 0; i < kLoadsB; ++i)
      load_to_lds(bbuf, b + (w * kLoadsB + i) * 8 * kStep, in ? bo[i] : kOOB, k);
    // the loads go out before the work that hides them
    __builtin_amdgcn_sched_barrier(0);
  };

  i32x16 acc[MT][NT] = {};
  const int ra = (w / WN) * (BM / WM) + c, rb = (w % WN) * (BN / WN) + c;
  auto work = [&](const int8_t* a, const int8_t* b) {
#pragma unroll
    for (int k = 0; k < kStep / 32; ++k) {
      i32x4 x[MT], y[NT];
#pragma unroll
      for (int i = 0; i < MT; ++i)
        x[i] = *reinterpret_cast<const i32x4*>(a + (ra + 32 * i) * kStep + 16 * ((2 * k + g) ^ (c & 7)));
#pragma unroll
      for (int j = 0; j < NT; ++j)
        y[j] = *reinterpret_cast<const i32x4*>(b + (rb + 32 * j) * kStep + 16 * ((2 * k + g) ^ (c & 7)));
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[i], y[j], acc[i][j], 0, 0, 0);
    }
  };
  // the buffer that is waited for is complete in every wave, and the other one
  // is no longer read, behind this
  auto ready = [] {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };

  const int steps = (p.K + kStep - 1) / kStep;
  fetch(a0, b0, 0);
  for (int s = 0; s + 1 < steps; s += 2) {
    ready();
    fetch(a1, b1, (s + 1) * kStep);
    work(a0, b0);
    ready();
    fetch(a0, b0, (s + 2) * kStep);  // behind the last step: zeros, from no memory
    work(a1, b1);
  }
  if (steps % 2) {
    ready();
    work(a0, b0);
  }

  Out* const out = static_cast<Out*>(p.out);
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int n = n0 + rb + 32 * j;
    const bool in = n < p.N;
    const float sw = in ? p.w_scale[n] : 0.f, bias = in && p.bias ? p.bias[n] : 0.f;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int m = m0 + ra - c + 32 * i + 8 * (e / 4) + 4 * g + e % 4;
        if (in && m < p.M) out[m * p.out_stride + n] = finish<Out>(acc[i][j][e], p.a_scale[m], sw, bias);
      }
  }
}

template <typename Out, int BM, int BN, int WM, int WN>
hipError_t tiles(const MatmulArgs& p, hipStream_t s) {
  const int64_t tm = (p.M + BM - 1) / BM, tn = (int64_t(p.N) + BN - 1) / BN;
  const int64_t groups = (tm * tn + kXcds - 1) / kXcds * kXcds;
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_matmul_tile<Out, BM, BN, WM, WN>), dim3(uint32_t(groups)), dim3(WM * WN * kWave), 0, s, p,
                     int(tm), int(tn));
  return hipGetLastError();
}
template <typename Out, int MT, int NT>
hipError_t skinny(const MatmulArgs& p, hipStream_t s) {
  hipLaunchKernelGGL((k_matmul_skinny<Out, MT, NT>), dim3((p.N + 16 * NT - 1) / (16 * NT), (p.M + 16 * MT - 1) / (16 * MT)),
                     dim3(kSkinnyWaves * kWave), 0, s, p);
  return hipGetLastError();
}
template <typename Out>
hipError_t matmul(const MatmulArgs& p, hipStream_t s) {
  if (p.M <= 16) return skinny<Out, 1, 1>(p, s);
  if (p.M <= 32) return skinny<Out, 2, 1>(p, s);
  if (p.M <= 64) return skinny<Out, 4, 1>(p, s);
  if (p.M <= 256) return skinny<Out, 4, 2>(p, s);
  const int64_t big = int64_t((p.M + 255) / 256) * ((p.N + 255) / 256);
  if (big >= 2 * kCUs) return tiles<Out, 256, 256, 2, 4>(p, s);
  return tiles<Out, 128, 128, 2, 2>(p, s);
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
  return out_dtype == WZ_BF16 ? matmul<uint16_t>(p, s) : matmul<float>(p, s);
}

}  // namespace wz
