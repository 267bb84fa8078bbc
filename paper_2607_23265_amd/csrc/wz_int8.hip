// Rows to 8-bit integers and their product with weights held the same way
// (wz_quantize_rows, wz_matmul_int).
#include <cmath>

#include "wz_serve.h"

namespace wz {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef u32x4 u32x4_of_2 __attribute__((aligned(2)));
typedef u32x4 u32x4_of_4 __attribute__((aligned(4)));

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

// ---------------------------------------------------------------------------
// The product
// ---------------------------------------------------------------------------

// One element of the result, in the order the header states.
template <typename Out>
__device__ __forceinline__ Out finish(int acc, float sa, float sw, float bias) {
  const float v = float(acc) * sa * sw + bias;
  if constexpr (sizeof(Out) == 2) return __builtin_bit_cast(uint16_t, __bf16(v));
  else return v;
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
// Tiles of BM x BN, WM x WN waves, 128 bytes of k at a time through ST stages of
// LDS that the loads write directly, ST - 1 stages ahead of the work.  KS such
// groups of waves take the steps in turn and add up their integers at the end.
// Chunks of 16 bytes are exchanged within a row by the row's number, so that
// sixteen lanes that read sixteen rows hit all 64 banks; the loads' lanes fetch
// in that order.
constexpr int KB = 128;  // bytes of a row in a stage
template <typename Out, int BM, int BN, int WM, int WN, int ST, int KS>
__global__ __launch_bounds__(WM* WN* KS* kWave) void k_matmul_tile(MatmulArgs p, int tiles_m, int tiles_n) {
  constexpr int kWaves = WM * WN, MT = BM / WM / 32, NT = BN / WN / 32;
  constexpr int kChunks = KB / 16, kLoadRows = kWave / kChunks;  // chunks of a row, rows of one load
  constexpr int kLoadsA = BM / kLoadRows / kWaves, kLoadsB = BN / kLoadRows / kWaves;
  static_assert(BM % (WM * 32) == 0 && BN % (WN * 32) == 0 &&
                    BM % (kLoadRows * kWaves) == 0 && BN % (kLoadRows * kWaves) == 0, "");
  constexpr int kStage = (BM + BN) * KB;
  __shared__ __align__(16) int8_t lds[ST * KS * kStage];  // [ST][KS][rows of a, then of w][KB]
  const int lane = __lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int w = wave % kWaves, group = wave / kWaves, c = lane & 31, g = lane >> 5;
  auto exchange = [](int row) { return row >> 1 & 7; };

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
  const int lr = lane / kChunks;  // this lane's row of a load
  i32x4 abuf = descriptor(p.a + int64_t(m0) * p.a_stride, min(BM, p.M - m0) * int(p.a_stride));
  i32x4 bbuf = descriptor(p.w + int64_t(n0) * p.w_stride, min(BN, p.N - n0) * int(p.w_stride));
  // a scalar register that the vector unit wrote may be a load's descriptor
  // five instructions later; the compiler does not look into the assembly
  asm volatile("s_nop 4" : "+s"(abuf), "+s"(bbuf));
  int ao[kLoadsA], bo[kLoadsB], ac[kLoadsA], bc[kLoadsB];  // offsets, and bytes within the step
#pragma unroll
  for (int i = 0; i < kLoadsA; ++i) {
    const int row = (w * kLoadsA + i) * kLoadRows + lr;
    ac[i] = 16 * ((lane % kChunks) ^ exchange(row)), ao[i] = row * int(p.a_stride) + ac[i];
  }
#pragma unroll
  for (int i = 0; i < kLoadsB; ++i) {
    const int row = (w * kLoadsB + i) * kLoadRows + lr;
    bc[i] = 16 * ((lane % kChunks) ^ exchange(row)), bo[i] = row * int(p.w_stride) + bc[i];
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
      load_to_lds(bbuf, to + BM * KB + (w * kLoadsB + x) * 1024, k + bc[x] < p.K ? bo[x] : kOOB, step);
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
  // them 16 bytes a lane, whole lines of the result (or half lines).
  constexpr int kUnitBytes = kWaves * 32 * 128 <= (BM + BN) * KB && BN / WN * sizeof(Out) >= 128 ? 128 : 64;
  constexpr int kUnit = kUnitBytes / sizeof(Out);  // columns of a unit
  constexpr int kUnitChunks = kUnit * sizeof(Out) / 16, kPer = 16 / sizeof(Out);  // 16-byte chunks of a row, elements
  static_assert(kWaves * 32 * kUnit * sizeof(Out) <= (BM + BN) * KB && BN / WN % kUnit == 0, "");
  Out* const out = static_cast<Out*>(p.out);
  Out* const unit = reinterpret_cast<Out*>(lds) + w * 32 * kUnit;
  auto place = [&](int row, int chunk) {
    return unit + row * kUnit + kPer * (chunk ^ (kUnitChunks == 8 ? row >> 1 & 7 : row >> 2 & 3));
  };
  float* const wsc = reinterpret_cast<float*>(lds + KS * kStage);  // [BN] scales, [BN] biases
  const int mw = m0 + (w / WN) * (BM / WM), nt = (w % WN) * (BN / WN);
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
    const int n = min(n0 + i, p.N - 1);
    wsc[i] = p.w_scale[n], wsc[BN + i] = p.bias ? p.bias[n] : 0.f;
  }
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const float sa = mw + 32 * i + c < p.M ? p.a_scale[mw + 32 * i + c] : 0.f;
#pragma unroll
    for (int u = 0; u < BN / WN; u += kUnit) {
#pragma unroll
      for (int col = 0; col < kUnit; col += 8) {
        const int j = (u + col) / 32, q = (u + col) % 32 / 8;
        const f32x4 sw = *reinterpret_cast<const f32x4*>(wsc + nt + u + col + 4 * g);
        const f32x4 bias = *reinterpret_cast<const f32x4*>(wsc + BN + nt + u + col + 4 * g);
        Out y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = finish<Out>(acc[i][j][4 * q + e], sa, sw[e], bias[e]);
        Out* to = place(c, (col + 4 * g) / kPer) + (col + 4 * g) % kPer;
        if constexpr (sizeof(Out) == 2)
          *reinterpret_cast<u32x2*>(to) = u32x2{y[0] | uint32_t(y[1]) << 16, y[2] | uint32_t(y[3]) << 16};
        else *reinterpret_cast<f32x4*>(to) = f32x4{y[0], y[1], y[2], y[3]};
      }
      // rows of the result may start at any element: stores of 16 bytes that
      // need no more than its alignment
      typedef std::conditional_t<sizeof(Out) == 2, u32x4_of_2, u32x4_of_4> loose;
      const int rows = min(32, p.M - (mw + 32 * i)), cols = min(kUnit, p.N - (n0 + nt + u));
      Out* const to = out + int64_t(mw + 32 * i) * p.out_stride + n0 + nt + u;
#pragma unroll
      for (int x = 0; x < 32 * kUnitChunks; x += kWave) {
        const int row = (x + lane) / kUnitChunks, chunk = (x + lane) % kUnitChunks;
        const u32x4 v = *reinterpret_cast<const u32x4*>(place(row, chunk));
        Out* const at = to + row * p.out_stride + kPer * chunk;
        if (row < rows && kPer * chunk + kPer <= cols) {
          *reinterpret_cast<loose*>(at) = v;
        } else if (row < rows) {
          for (int e = 0; e < cols - kPer * chunk; ++e) at[e] = place(row, chunk)[e];
        }
      }
    }
  }
}

template <typename Out, int BM, int BN, int WM, int WN, int ST, int KS>
hipError_t tiles(const MatmulArgs& p, hipStream_t s) {
  const int64_t tm = (p.M + BM - 1) / BM, tn = (int64_t(p.N) + BN - 1) / BN;
  const int64_t groups = (tm * tn + kXcds - 1) / kXcds * kXcds;
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_matmul_tile<Out, BM, BN, WM, WN, ST, KS>), dim3(uint32_t(groups)), dim3(WM * WN * KS * kWave),
                     0, s, p, int(tm), int(tn));
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
template <typename Out>
struct Tile {
  int bm, bn;
  double fixed, ends, steps;
  int at_once;
  hipError_t (*run)(const MatmulArgs&, hipStream_t);

  int64_t columns(const MatmulArgs& p) const { return (int64_t(p.N) + bn - 1) / bn; }
  int64_t count(const MatmulArgs& p) const { return (int64_t(p.M) + bm - 1) / bm * columns(p); }
  double time(const MatmulArgs& p, double rounds) const { return fixed + rounds * (ends + steps * (p.K / 3584.)); }
  double time(const MatmulArgs& p) const {
    const double rounds = double(count(p)) / (kCUs * at_once), full = std::floor(rounds), f = rounds - full;
    return time(p, full + (f > 0 ? 0.6 + 0.4 * f : 0.));
  }
};

template <typename Out>
hipError_t matmul(const MatmulArgs& p, hipStream_t s) {
  // Where 32 x 32 or 64 x 32 tiles are no more than the CUs, a product waits for
  // its steps of K one after the other: four groups of waves share those of a 32
  // x 32 tile, two those of a 64 x 32 tile (a row of 4608 columns: 6.1 us, in 64 x
  // 64 tiles 8.8; 64 rows 7.7 against 9.2; 300 x 256 x 8192: 9.1, 11.3 and 13.9 in
  // tiles of 32 x 32, 64 x 32 and 64 x 64).
  auto count = [&](int bm, int bn) { return (int64_t(p.M) + bm - 1) / bm * ((int64_t(p.N) + bn - 1) / bn); };
  if (count(32, 32) <= kCUs) return tiles<Out, 32, 32, 1, 1, 4, 4>(p, s);
  if (count(64, 32) <= kCUs) return tiles<Out, 64, 32, 2, 1, 4, 2>(p, s);
  static constexpr Tile<Out> kTiles[] = {
      {64, 64, 3.9, 1.0, 4.7, 1, tiles<Out, 64, 64, 2, 2, 4, 1>},
      {128, 64, 4.3, 1.35, 8.3, 1, tiles<Out, 128, 64, 2, 2, 3, 1>},
      {128, 128, 3.1, 3.7, 14.0, 1, tiles<Out, 128, 128, 2, 2, 3, 1>},
      {128, 128, 3.7, 3.9, 26.0, 2, tiles<Out, 128, 128, 2, 2, 2, 1>},
      {192, 128, 2.5, 3.8, 19.6, 1, tiles<Out, 192, 128, 2, 4, 3, 1>},
      {256, 256, 8.0, 5.0, 44.6, 1, tiles<Out, 256, 256, 2, 4, 2, 1>},
  };
  auto fastest = [&](const MatmulArgs& q) {
    const Tile<Out>* best = kTiles;
    for (const Tile<Out>& t : kTiles)
      if (t.time(q) < best->time(q)) best = &t;
    return best;
  };
  // Rows of tiles that fill whole rounds, and what is left in tiles that fit it
  // better, as a second launch, where that is faster than a last round of a few
  // tiles (9459 x 14336: 2072 tiles of 256 x 256 are 8 rounds and 24 tiles).
  const Tile<Out>* const whole = fastest(p);
  double best = whole->time(p);
  const Tile<Out>* first = nullptr;
  int rows = 0;
  for (const Tile<Out>& t : kTiles) {
    const int64_t at_once = kCUs * t.at_once, rounds = t.count(p) / at_once;
    const int64_t full = rounds * at_once / t.columns(p) * t.bm;
    if (full <= 0 || full >= p.M) continue;
    MatmulArgs rest = p;
    rest.M = p.M - int(full);
    const double time = t.time(p, double(rounds)) + fastest(rest)->time(rest);
    if (time < best) best = time, first = &t, rows = int(full);
  }
  if (!first) return whole->run(p, s);
  MatmulArgs part = p;
  part.M = rows;
  const hipError_t e = first->run(part, s);
  if (e != hipSuccess) return e;
  part.M = p.M - rows;
  part.a += rows * p.a_stride, part.a_scale += rows;
  part.out = static_cast<Out*>(p.out) + rows * p.out_stride;
  return fastest(part)->run(part, s);
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
