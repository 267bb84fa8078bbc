// The product of 8-bit integers in tiles, for the entry points that differ in
// what becomes of its sums (wz_matmul_int, wz_matmul_int_epilogue, wz_gated_int).
#pragma once

#include <cmath>

#include "wz_serve.h"

namespace wz {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef u32x4 u32x4_of_2 __attribute__((aligned(2)));
typedef u32x4 u32x4_of_4 __attribute__((aligned(4)));

// What becomes of a tile's sums: scaled, with a bias (kPlain); and an activation
// and a residual (kRich); or activation and product of two weights' sums (kGated).
enum Epilogue { kPlain, kRich, kGated };

// One element of the result, in the order the header states.
__device__ __forceinline__ float scaled(int acc, float sa, float sw, float bias) { return float(acc) * sa * sw + bias; }
template <typename Out>
__device__ __forceinline__ Out rounded(float v) {
  if constexpr (sizeof(Out) == 2) return __builtin_bit_cast(uint16_t, __bf16(v));
  else return v;
}

// Activations in three forms, so that an epilogue is compiled three times and
// not once for each: x or max(x, 0); x s(z) with s(z) = 1 / (1 + exp(-z)) and z an
// odd cubic of x (silu: z = x; the tanh form of gelu, for (1 + tanh(z / 2)) / 2 =
// s(z): z = 2 sqrt(2/pi) (x + 0.044715 x^3)); and the error function.
struct ActLinear {
  float floor;  // -inf: none
  __device__ __forceinline__ float operator()(float x) const { return x < floor ? floor : x; }  // (NaN stays)
};
struct ActSigmoid {
  float c1, c3;  // of -z log2(e)
  __device__ __forceinline__ float operator()(float x) const {
    // (an infinite square times silu's c3 of zero would be no number)
    return x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * fmaf(c3, fminf(x * x, 1e30f), c1)));
  }
};
// x (1 + erf(x / sqrt 2)) / 2 = max(x, 0) - |x| g(|x|) with g(a) = erfc(a / sqrt 2) / 2 = P(t)
// exp(-a^2 / 2), t = 1 / (1 + 0.34375 a).  P, of degree 9, is the least largest relative
// error of a polynomial without a constant term over 0 <= a <= 16 (3.6e-8; 7.2e-8 with its
// coefficients rounded to fp32), found by reweighted least squares: g is good to fp32 in its
// tail too, where 1 + erf cancels (tests/test_gpu_serve_gelu.py has the bound).  12544 x 3584 x
// 1152 to bf16, to fp32, and x 576 to bf16: 83, 91 and 62 us on one card; with a published
// form of degree 5, within 1.5e-7 of erfc, 81, 89 and 60; with the library's erff 100, 107, 78.
struct ActErf {
  __device__ __forceinline__ float operator()(float x) const {
    const float a = fminf(fabsf(x), 16.f);  // (beyond that nothing is left of the second term)
    const float t = __builtin_amdgcn_rcpf(fmaf(a, 0.34375f, 1.f));
    float y = fmaf(t, -0.026958352f, 0.139933586f);
    y = fmaf(t, y, -0.26410526f);
    y = fmaf(t, y, 0.182793453f);
    y = fmaf(t, y, -0.0341064557f);
    y = fmaf(t, y, 0.110624172f);
    y = fmaf(t, y, 0.117213458f);
    y = fmaf(t, y, 0.137482643f);
    y = fmaf(t, y, 0.13712278f) * t;
    y *= a * __builtin_amdgcn_exp2f(a * a * (-0.5f * 1.44269504088896341f));
    return (x < 0.f ? 0.f : x) - y;  // (NaN stays)
  }
};
template <typename F>
__device__ __forceinline__ void with_activation(int activation, F f) {
  constexpr float kLog2e = 1.44269504088896341f, kTanh = 2 * 0.797884560802865356f;  // 2 sqrt(2 / pi)
  if (activation == WZ_ACT_SILU || activation == WZ_ACT_GELU_TANH) {
    const bool silu = activation == WZ_ACT_SILU;
    f(ActSigmoid{silu ? -kLog2e : -kLog2e * kTanh, silu ? 0.f : -kLog2e * kTanh * 0.044715f});
  } else if (activation == WZ_ACT_GELU) {
    f(ActErf{});
  } else {
    f(ActLinear{activation == WZ_ACT_RELU ? 0.f : -INFINITY});
  }
}

// 16 bytes a lane from a buffer to LDS, lane after lane from `to` on (the
// same in every lane); zeros for an offset behind the buffer's end.  It has no
// register for a result.  As assembly because the compiler, which cannot tell
// stages apart once more than a few loads are under way, would otherwise wait
// for all of them before every read of LDS; wait_loads() is the only wait.
__device__ __forceinline__ void load_to_lds(i32x4 buffer, uint32_t to, int offset, int uniform) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(offset),
               "s"(buffer), "s"(uniform)
               : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}
// A buffer's descriptor in scalar registers.
__device__ __forceinline__ i32x4 descriptor(const void* base, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  return i32x4{__builtin_amdgcn_readfirstlane(int(uint32_t(a))),
               __builtin_amdgcn_readfirstlane(int(uint32_t(a >> 32) & 0xffffu)),
               __builtin_amdgcn_readfirstlane(int(bytes)), kBufWord3};
}

// All but the wave's last N loads from memory, and all its reads of LDS, are done.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// Measured: 9459 x 14336 x 3584 in 442 us (2.2 POP/s, as the library's 8192^3
// product; 21 us more for the rows), 1286 x 4608 x 3584 in 25.9, 64 rows in 7.7.
// The matrix cores are busy for 58 % of the large product's cycles (at 1.9 GHz),
// LDS for 26 %.
//
// Tiles of BM x BN, WM x WN waves, KB bytes of k at a time through ST stages of
// LDS that the loads write directly, ST - 1 stages ahead of the work.  KS such
// groups of waves take the steps in turn and add up their integers at the end.
// Chunks of 16 bytes are exchanged within a row by the row's number, so that
// sixteen lanes that read sixteen rows hit all 64 banks; the loads' lanes fetch
// in that order.
//
// kGated: a tile's BN rows of weights are 16 of the gate and 16 of the other
// projection in turn, so that a lane has both sums of an element, in eight
// registers of the same fragment, and neither leaves the registers.
//
// KB = 64: half of the LDS, and registers for three tiles on a CU.
template <typename Out, int BM, int BN, int WM, int WN, int ST, int KS, int EPI, int KB>
__global__ __launch_bounds__(WM* WN* KS* kWave, KB == 64 ? 3 : 1) void k_matmul_tile(MatmulArgs p, int tiles_m, int tiles_n) {
  constexpr int kWaves = WM * WN, MT = BM / WM / 32, NT = BN / WN / 32;
  constexpr int kChunks = KB / 16, kLoadRows = kWave / kChunks;  // chunks of a row, rows of one load
  constexpr int kLoadsA = BM / kLoadRows / kWaves, kLoadsB = BN / kLoadRows / kWaves;
  static_assert(BM % (WM * 32) == 0 && BN % (WN * 32) == 0 &&
                    BM % (kLoadRows * kWaves) == 0 && BN % (kLoadRows * kWaves) == 0, "");
  constexpr int kStage = (BM + BN) * KB;
  __shared__ __align__(16) int8_t lds[ST * KS * kStage];  // [ST][KS][rows of a, then of w][KB]
  const int lane = __lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int w = wave % kWaves, group = wave / kWaves, c = lane & 31, g = lane >> 5;
  auto exchange = [](int row) { return KB == 128 ? row >> 1 & 7 : row >> 2 & 3; };

  // Workgroups go to the XCDs in turn: each XCD gets a run of tiles that lie
  // together (columns of 8 row tiles), whose rows and weights its L2 holds.
  const int tiles = tiles_m * tiles_n, per = (tiles + kXcds - 1) / kXcds;
  const int t = (blockIdx.x % kXcds) * per + blockIdx.x / kXcds;
  if (blockIdx.x / kXcds >= per || t >= tiles) return;
  constexpr int kBand = 8;
  const int band = t / (kBand * tiles_n), in_band = t % (kBand * tiles_n);
  const int band_rows = min(kBand, tiles_m - band * kBand);
  const int tm = band * kBand + in_band % band_rows, tn = in_band / band_rows;
  constexpr int kCols = EPI == kGated ? BN / 2 : BN;  // columns of the result
  const int m0 = tm * BM, n0 = tn * kCols;
  // a row of a tile's weights: its column of the result, and whether it is the gate's
  auto column = [](int row) { return EPI == kGated ? (row >> 5) * 16 + (row & 15) : row; };
  auto second = [](int row) { return EPI == kGated && (row & 16); };

  // a row behind the last one is behind its buffer's end and reads as zeros;
  // so is, by its offset, what lies behind the end of a row
  const int lr = lane / kChunks;  // this lane's row of a load
  i32x4 abuf = descriptor(p.a + int64_t(m0) * p.a_stride, min(BM, p.M - m0) * int(p.a_stride));
  i32x4 bbuf = descriptor(p.w + int64_t(n0) * p.w_stride, min(kCols, p.N - n0) * int(p.w_stride));
  i32x4 ubuf = bbuf;
  if constexpr (EPI == kGated)
    ubuf = descriptor(p.w2 + int64_t(n0) * p.w2_stride, min(kCols, p.N - n0) * int(p.w2_stride));
  // a scalar register that the vector unit wrote may be a load's descriptor
  // five instructions later; the compiler does not look into the assembly
  asm volatile("s_nop 4" : "+s"(abuf), "+s"(bbuf), "+s"(ubuf));
  int ao[kLoadsA], bo[kLoadsB], ac[kLoadsA], bc[kLoadsB];  // offsets, and bytes within the step
#pragma unroll
  for (int i = 0; i < kLoadsA; ++i) {
    const int row = (w * kLoadsA + i) * kLoadRows + lr;
    ac[i] = 16 * ((lane % kChunks) ^ exchange(row)), ao[i] = row * int(p.a_stride) + ac[i];
  }
#pragma unroll
  for (int i = 0; i < kLoadsB; ++i) {
    const int row = (w * kLoadsB + i) * kLoadRows + lr;
    bc[i] = 16 * ((lane % kChunks) ^ exchange(row));
    bo[i] = column(row) * int(second(row) ? p.w2_stride : p.w_stride) + bc[i];
  }
  const uint32_t base = lds_address(lds) + group * kStage;
  auto fetch = [&](int i, int s) {  // step s to stage i
    const int k = (s * KS + group) * KB;
    const uint32_t to = base + i * KS * kStage;
    const int step = k < p.K ? k : 0;  // behind the last step every lane's offset is out of range by itself
#pragma unroll
    for (int x = 0; x < kLoadsA; ++x)
      load_to_lds(abuf, to + (w * kLoadsA + x) * 1024, k + ac[x] < p.K ? ao[x] : kOOB, step);
#pragma unroll
    for (int x = 0; x < kLoadsB; ++x)
      load_to_lds(second((w * kLoadsB + x) * kLoadRows) ? ubuf : bbuf, to + BM * KB + (w * kLoadsB + x) * 1024,
                  k + bc[x] < p.K ? bo[x] : kOOB, step);
  };

  i32x16 acc[MT][NT] = {};
  const int ra = (w / WN) * (BM / WM) + c, rb = (w % WN) * (BN / WN) + c, ex = exchange(c);
  // Two sets of fragments: one is read while the products of the other run.
  struct Set {
    i32x4 x[MT], y[NT];
  } even, odd;
  auto read = [&](const int8_t* a, int k, Set& f) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
      f.x[i] = *reinterpret_cast<const i32x4*>(a + (ra + 32 * i) * KB + 16 * ((2 * k + g) ^ ex));
#pragma unroll
    for (int j = 0; j < NT; ++j)
      f.y[j] = *reinterpret_cast<const i32x4*>(a + BM * KB + (rb + 32 * j) * KB + 16 * ((2 * k + g) ^ ex));
    __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply = [&](const Set& f) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.y[j], f.x[i], acc[i][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  // Step s, in stage `now`: behind the barrier its loads, which every wave waits
  // for, are complete, and the stage that the next loads go to (step s - 1's) is
  // no longer read: its last fragments are in registers, and their products
  // hide this step's first reads.  Behind the last step the loads are of
  // zeros, from no memory.
  const int steps = (p.K + KB * KS - 1) / (KB * KS);
#pragma unroll
  for (int i = 0; i < MT; ++i) odd.x[i] = i32x4{};  // the first products of all are of zeros
#pragma unroll
  for (int j = 0; j < NT; ++j) odd.y[j] = i32x4{};
#pragma unroll
  for (int i = 0; i < ST - 1; ++i) fetch(i, i);
  auto step = [&](int s, int now, int next) {
    wait_loads<(ST - 2) * (kLoadsA + kLoadsB)>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    fetch(next, s + ST - 1);
    const int8_t* const at = lds + (now * KS + group) * kStage;
#pragma unroll
    for (int k = 0; k < KB / 32; k += 2) {
      read(at, k, even);
      multiply(odd);
      read(at, k + 1, odd);
      multiply(even);
    }
  };
  int s = 0;
  for (; s + ST <= steps; s += ST) {  // (with its stages known, a step's addresses need no arithmetic)
#pragma unroll
    for (int i = 0; i < ST; ++i) step(s + i, i, (i + ST - 1) % ST);
  }
  for (int i = 0; s + i < steps; ++i) step(s + i, i, i == 0 ? ST - 1 : i - 1);
  multiply(odd);
  wait_loads<0>();  // no load may write LDS behind the workgroup's end

  // The weights are the left operand, so a lane has four columns of one row
  // together.  A wave turns units of 32 rows by 128 bytes in LDS and stores
  // them 16 bytes a lane, whole lines of the result (or halves or quarters).
  constexpr int kWaveCols = EPI == kGated ? BN / WN / 2 : BN / WN;
  constexpr int kMostBytes = kWaveCols * int(sizeof(Out));
  constexpr int kUnitBytes =
      kWaves * 32 * 128 <= (BM + BN) * KB && kMostBytes >= 128 ? 128 : kMostBytes >= 64 ? 64 : 32;
  constexpr int kUnit = kUnitBytes / sizeof(Out);  // columns of a unit
  constexpr int kUnitChunks = kUnit * sizeof(Out) / 16, kPer = 16 / sizeof(Out);  // 16-byte chunks of a row, elements
  static_assert(kWaves * 32 * kUnit * sizeof(Out) <= (BM + BN) * KB && kWaveCols % kUnit == 0, "");
  Out* const out = static_cast<Out*>(p.out);
  Out* const unit = reinterpret_cast<Out*>(lds) + w * 32 * kUnit;
  auto place = [&](int row, int chunk) {
    const int x = kUnitChunks == 8 ? row >> 1 & 7 : kUnitChunks == 4 ? row >> 2 & 3 : row >> 3 & 1;
    return unit + row * kUnit + kPer * (chunk ^ x);
  };
  float* const wsc = reinterpret_cast<float*>(lds + KS * kStage);  // [BN] scales, [BN] biases
  const int mw = m0 + (w / WN) * (BM / WM), nt = (w % WN) * kWaveCols;
  const int wt = (w % WN) * (BN / WN);  // the wave's first row of weights
  __syncthreads();  // no wave reads its stages any more
  if constexpr (KS > 1) {
    static_assert((KS - 1) * kWaves * MT * NT * 4096 <= KS * kStage, "");
    i32x4* const sums = reinterpret_cast<i32x4*>(lds + KS * kStage) + w * (MT * NT * 4 * kWave) + lane;
    auto each = [&](auto f) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) f(acc[i][j], q, ((i * NT + j) * 4 + q) * kWave);
    };
    if (group > 0)
      each([&](i32x16& x, int q, int at) {
        sums[(group - 1) * kWaves * MT * NT * 4 * kWave + at] =
            i32x4{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
      });
    __syncthreads();
    if (group == 0)
      for (int k = 0; k < KS - 1; ++k)
        each([&](i32x16& x, int q, int at) {
          const i32x4 y = sums[k * kWaves * MT * NT * 4 * kWave + at];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[4 * q + e] += y[e];
        });
    __syncthreads();
  }
  for (int i = threadIdx.x; i < BN; i += KS * kWaves * kWave) {
    const int n = min(n0 + column(i), p.N - 1);
    const float* const s = second(i) ? p.w2_scale : p.w_scale;
    const float* const b = second(i) ? p.bias2 : p.bias;
    wsc[i] = s[n], wsc[BN + i] = b ? b[n] : 0.f;
  }
  __syncthreads();
  if (group > 0) return;
  // rows of the result may start at any element: accesses of 16 bytes that
  // need no more than its alignment
  typedef std::conditional_t<sizeof(Out) == 2, u32x4_of_2, u32x4_of_4> loose;
  constexpr int kMoves = (32 * kUnitChunks + kWave - 1) / kWave, kUnits = kWaveCols / kUnit;
  // Each 16-byte chunk of unit u of fragment row i: f(its number, row, chunk, offset
  // in a matrix of that stride, elements that exist).
  auto chunks = [&](int i, int u, int64_t stride, auto f) {
    const int rows = min(32, p.M - (mw + 32 * i)), cols = min(kUnit, p.N - (n0 + nt + u));
    const int64_t first = int64_t(mw + 32 * i) * stride + n0 + nt + u;
#pragma unroll
    for (int x = 0; x < kMoves; ++x) {
      const int row = (x * kWave + lane) / kUnitChunks, chunk = (x * kWave + lane) % kUnitChunks;
      if (row < rows) f(x, row, chunk, first + row * stride + kPer * chunk, min(cols - kPer * chunk, kPer));
    }
  };
  auto finish = [&](auto act) {
    // a unit of the residual is asked for before the unit that goes before it is worked on
    const Out* const residual = EPI == kRich ? static_cast<const Out*>(p.residual) : nullptr;
    u32x4 res[2][kMoves] = {};
    auto ask = [&](int n) {
      chunks(n / kUnits, n % kUnits * kUnit, p.residual_stride, [&](int x, int, int, int64_t at, int there) {
        if (there == kPer) res[n & 1][x] = *reinterpret_cast<const loose*>(residual + at);
      });
    };
    if (residual) ask(0);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const float sa = mw + 32 * i + c < p.M ? p.a_scale[mw + 32 * i + c] : 0.f;
#pragma unroll
      for (int u = 0; u < kWaveCols; u += kUnit) {
        const int n = i * kUnits + u / kUnit;
        if (residual) {
          if (n + 1 < MT * kUnits) ask(n + 1);
          chunks(i, u, p.residual_stride, [&](int x, int row, int chunk, int64_t at, int there) {
            if (there == kPer) {
              *reinterpret_cast<u32x4*>(place(row, chunk)) = res[n & 1][x];
            } else {
              for (int e = 0; e < there; ++e) place(row, chunk)[e] = residual[at + e];
            }
          });
        }
#pragma unroll
        for (int col = 0; col < kUnit; col += 8) {
          float v[4];
          Out* const to = place(c, (col + 4 * g) / kPer) + (col + 4 * g) % kPer;
          if constexpr (EPI == kGated) {
            const int j = (u + col) / 16, q = (u + col) % 16 / 8, at = wt + 32 * j + 8 * q + 4 * g;
            const f32x4 sg = *reinterpret_cast<const f32x4*>(wsc + at);
            const f32x4 su = *reinterpret_cast<const f32x4*>(wsc + at + 16);
            const f32x4 bg = *reinterpret_cast<const f32x4*>(wsc + BN + at);
            const f32x4 bu = *reinterpret_cast<const f32x4*>(wsc + BN + at + 16);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] = act(scaled(acc[i][j][4 * q + e], sa, sg[e], bg[e])) *
                     scaled(acc[i][j][8 + 4 * q + e], sa, su[e], bu[e]);
          } else {
            const int j = (u + col) / 32, q = (u + col) % 32 / 8;
            const f32x4 sw = *reinterpret_cast<const f32x4*>(wsc + nt + u + col + 4 * g);
            const f32x4 bias = *reinterpret_cast<const f32x4*>(wsc + BN + nt + u + col + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = act(scaled(acc[i][j][4 * q + e], sa, sw[e], bias[e]));
          }
          if (residual) {
            if constexpr (sizeof(Out) == 2) {
              const u32x2 r = *reinterpret_cast<const u32x2*>(to);
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] += e % 2 ? bf16_hi(r[e / 2]) : bf16_lo(r[e / 2]);
            } else {
              const f32x4 r = *reinterpret_cast<const f32x4*>(to);
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] += r[e];
            }
          }
          Out y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = rounded<Out>(v[e]);
          if constexpr (sizeof(Out) == 2)
            *reinterpret_cast<u32x2*>(to) = u32x2{y[0] | uint32_t(y[1]) << 16, y[2] | uint32_t(y[3]) << 16};
          else *reinterpret_cast<f32x4*>(to) = f32x4{y[0], y[1], y[2], y[3]};
        }
        chunks(i, u, p.out_stride, [&](int, int row, int chunk, int64_t at, int there) {
          const u32x4 v = *reinterpret_cast<const u32x4*>(place(row, chunk));
          if (there == kPer) {
            *reinterpret_cast<loose*>(out + at) = v;
          } else {
            for (int e = 0; e < there; ++e) out[at + e] = place(row, chunk)[e];
          }
        });
      }
    }
  };
  if constexpr (EPI == kPlain) finish([](float v) { return v; });
  else with_activation(p.activation, finish);
}

// Rows of weights that a product's tiles go over.
template <int EPI>
int64_t weight_rows(const MatmulArgs& p) { return EPI == kGated ? 2 * int64_t(p.N) : p.N; }

template <typename Out, int BM, int BN, int WM, int WN, int ST, int KS, int EPI, int KB = 128>
hipError_t tiles(const MatmulArgs& p, hipStream_t s) {
  const int64_t tm = (p.M + BM - 1) / BM, tn = (weight_rows<EPI>(p) + BN - 1) / BN;
  const int64_t groups = (tm * tn + kXcds - 1) / kXcds * kXcds;
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_matmul_tile<Out, BM, BN, WM, WN, ST, KS, EPI, KB>), dim3(uint32_t(groups)),
                     dim3(WM * WN * KS * kWave), 0, s, p, int(tm), int(tn));
  return hipGetLastError();
}

// A tile's time, measured (us): a launch takes `fixed`, and for every round of the
// CUs, which work on `at_once` tiles each, `ends` for the tiles' first loads and
// their results and `steps` for 3584 of K; the last round, with a share f of its
// tiles, takes 0.6 + 0.4 f of one (256 x 256 tiles: 41.3 us with 108, 57.6 with 256,
// 149 with 666).  Large tiles read LDS less for the same products, small ones fill
// the chip; three stages hide a step's loads behind two others where a CU has one
// tile (128 x 128: 20.8 us with three, 23.5 with two), and two leave room for a
// second tile (33.1 for both).
template <typename Out, int EPI>
struct Tile {
  int bm, bn;
  double fixed, ends, steps;
  int at_once;
  hipError_t (*run)(const MatmulArgs&, hipStream_t);

  int64_t columns(const MatmulArgs& p) const { return (weight_rows<EPI>(p) + bn - 1) / bn; }
  int64_t count(const MatmulArgs& p) const { return (int64_t(p.M) + bm - 1) / bm * columns(p); }
  // An activation's instructions, in a round's ends: 10 us with the error function for
  // 256 x 256 elements, where a second tile's products hide them 4.4 (12544 x 3584 x
  // 1152: 92 us in tiles of 256 x 256, 87 in two of 128 x 128 at a time, with an error
  // function of four instructions less; without one the first are the faster).
  double act(const MatmulArgs& p) const {
    if (EPI == kPlain || p.activation == WZ_ACT_NONE || p.activation == WZ_ACT_RELU) return 0;
    const double elements = at_once * bm * bn / 65536. * (EPI == kGated ? 0.5 : 1.);
    return (p.activation == WZ_ACT_GELU ? 10. : 5.) * (at_once > 1 ? 0.44 : 1.) * elements;
  }
  double time(const MatmulArgs& p, double rounds) const {
    return fixed + rounds * (ends + act(p) + steps * (p.K / 3584.));
  }
  double time(const MatmulArgs& p) const {
    const double rounds = double(count(p)) / (kCUs * at_once), full = std::floor(rounds), f = rounds - full;
    return time(p, full + (f > 0 ? 0.6 + 0.4 * f : 0.));
  }
};

template <typename Out, int EPI>
hipError_t matmul(const MatmulArgs& p, hipStream_t s) {
  // Where 32 x 32 or 64 x 32 tiles are no more than the CUs, a product waits for
  // its steps of K one after the other: four groups of waves share those of a 32
  // x 32 tile, two those of a 64 x 32 tile (a row of 4608 columns: 6.1 us, in 64 x
  // 64 tiles 8.8; 64 rows 7.7 against 9.2; 300 x 256 x 8192: 9.1, 11.3 and 13.9 in
  // tiles of 32 x 32, 64 x 32 and 64 x 64).
  auto count = [&](int bm, int bn) { return (int64_t(p.M) + bm - 1) / bm * ((weight_rows<EPI>(p) + bn - 1) / bn); };
  if (count(32, 32) <= kCUs) return tiles<Out, 32, 32, 1, 1, 4, 4, EPI>(p, s);
  if (count(64, 32) <= kCUs) return tiles<Out, 64, 32, 2, 1, 4, 2, EPI>(p, s);
  static constexpr Tile<Out, EPI> kTiles[] = {
      {64, 64, 3.9, 1.0, 4.7, 1, tiles<Out, 64, 64, 2, 2, 4, 1, EPI>},
      {128, 64, 4.3, 1.35, 8.3, 1, tiles<Out, 128, 64, 2, 2, 3, 1, EPI>},
      {128, 128, 3.1, 3.7, 14.0, 1, tiles<Out, 128, 128, 2, 2, 3, 1, EPI>},
      {128, 128, 3.7, 3.9, 26.0, 2, tiles<Out, 128, 128, 2, 2, 2, 1, EPI>},
      {192, 128, 2.5, 3.8, 19.6, 1, tiles<Out, 192, 128, 2, 4, 3, 1, EPI>},
      {256, 256, 8.0, 5.0, 44.6, 1, tiles<Out, 256, 256, 2, 4, 2, 1, EPI>},
  };
  // For few steps of K and an activation, whose instructions three tiles on a CU hide
  // better than two: gelu after 12544 x 3584 x 576 63 us, without this 74, x 1152 84 and
  // 93, silu 79 and 84; gated 6000 x 4304 x 576 52 and 64.  (Gelu, x 2304: 143 and 141.)
  auto each = [](auto f) {
    for (const Tile<Out, EPI>& t : kTiles) f(t);
    if constexpr (EPI != kPlain) {
      static constexpr Tile<Out, EPI> kThree{128, 128, 3.7, 3.5, 43.9, 3, tiles<Out, 128, 128, 2, 2, 3, 1, EPI, 64>};
      f(kThree);
    }
  };
  auto fastest = [&](const MatmulArgs& q) {
    const Tile<Out, EPI>* best = kTiles;
    each([&](const Tile<Out, EPI>& t) {
      if (t.time(q) < best->time(q)) best = &t;
    });
    return best;
  };
  // Rows of tiles that fill whole rounds, and what is left in tiles that fit it
  // better, as a second launch, where that is faster than a last round of a few
  // tiles (9459 x 14336: 2072 tiles of 256 x 256 are 8 rounds and 24 tiles).
  const Tile<Out, EPI>* const whole = fastest(p);
  double best = whole->time(p);
  const Tile<Out, EPI>* first = nullptr;
  int rows = 0;
  each([&](const Tile<Out, EPI>& t) {
    const int64_t at_once = kCUs * t.at_once, rounds = t.count(p) / at_once;
    const int64_t full = rounds * at_once / t.columns(p) * t.bm;
    if (full <= 0 || full >= p.M) return;
    MatmulArgs rest = p;
    rest.M = p.M - int(full);
    const double time = t.time(p, double(rounds)) + fastest(rest)->time(rest);
    if (time < best) best = time, first = &t, rows = int(full);
  });
  if (!first) return whole->run(p, s);
  MatmulArgs part = p;
  part.M = rows;
  const hipError_t e = first->run(part, s);
  if (e != hipSuccess) return e;
  part.M = p.M - rows;
  part.a += rows * p.a_stride, part.a_scale += rows;
  part.out = static_cast<Out*>(p.out) + rows * p.out_stride;
  if (p.residual) part.residual = static_cast<const Out*>(p.residual) + rows * p.residual_stride;
  return fastest(part)->run(part, s);
}

}  // namespace
}  // namespace wz
