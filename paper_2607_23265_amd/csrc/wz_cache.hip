// Appending to the 8-bit paged cache (wz_cache_append): rotation, scales,
// rounding and layout in one launch.
//
// A workgroup of the first part owns one page that receives tokens and one
// key/value head, so the page's scales need no other workgroup: it reads the
// new keys and values once into registers, takes their largest magnitudes,
// fixes both scales, moves what the page held to them if they grew, and
// writes codes.  Values are turned to [head_dim][page_size] through LDS.
// Workgroups behind those rotate the queries.
//
// Measured: 48 869 prompt tokens of eight sequences, 28 + 2 * 4 heads of 128, 851 MB
// in 162 us (5.3 TB/s, as a 1 GiB copy); a token each of 64 sequences in 5.0 us,
// three waits for memory in a row behind the launch.
#include "wz_serve.h"

namespace wz {
namespace {

constexpr int kThreads = 256;

// Eight consecutive elements as they lie in memory, and as fp32.
template <typename In>
struct Raw8 {
  u32x4 u[sizeof(In) / 2];
  __device__ __forceinline__ void load(const In* p) {
#pragma unroll
    for (int i = 0; i < int(sizeof(In) / 2); ++i) u[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(In) == 2) x[i] = i % 2 ? bf16_hi(u[0][i / 2]) : bf16_lo(u[0][i / 2]);
      else x[i] = __uint_as_float(u[i / 4][i % 4]);
    }
  }
};
template <typename In>
struct Raw4 {
  uint32_t u[sizeof(In)];
  __device__ __forceinline__ void load(const In* p) {
    if constexpr (sizeof(In) == 2) {
      const u32x2 v = *reinterpret_cast<const u32x2*>(p);
      u[0] = v[0], u[1] = v[1];
    } else {
      const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = v[i];
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(In) == 2) return i % 2 ? bf16_hi(u[i / 2]) : bf16_lo(u[i / 2]);
    else return __uint_as_float(u[i]);
  }
};

// A head's row is shared by D / 16 lanes with two chunks of eight elements
// each: lane j of the first rot_dim / 16 has the two halves of eight pairs
// (interleaved: two chunks of four pairs each), the others two chunks that are
// not rotated.
struct Chunks {
  int a, b;     // offsets in elements
  bool turned;  // whether they are
};
__device__ __forceinline__ Chunks chunks_of(const wz_rotation& r, int lane) {
  const int pairs = r.rot_dim / 16;
  if (lane < pairs && !r.interleaved) return Chunks{8 * lane, 8 * lane + r.rot_dim / 2, true};
  return Chunks{16 * lane, 16 * lane + 8, lane < pairs};
}

// The row of positions that frequency f goes by, and token t's position there.
__device__ __forceinline__ int section_of(const wz_rotation& r, int f) {
  return r.axes == 1 ? 0 : f < r.sections[0] ? 0 : f < r.sections[0] + r.sections[1] ? 1 : 2;
}
__device__ __forceinline__ int position_of(const wz_rotation& r, int tokens, int t, int axis) {
  return r.positions[int64_t(axis) * tokens + t];
}
// The cosines and sines of a lane's eight frequencies for token t; position: its
// position for the first of them, asked for earlier.
struct Angles {
  float c[8], s[8];
};
__device__ __forceinline__ void angles(const wz_rotation& r, int tokens, int t, int lane, int position, Angles& x) {
  const int half = r.rot_dim / 2, j = 8 * lane;
  auto row = [&](int p) { return r.table + int64_t(min(max(p, 0), r.max_pos - 1)) * r.rot_dim; };
  if (section_of(r, j) == section_of(r, j + 7)) {
    const float* p = row(position) + j;
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const f32x4 u = *reinterpret_cast<const f32x4*>(p + i), w = *reinterpret_cast<const f32x4*>(p + half + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.c[i + e] = u[e], x.s[i + e] = w[e];
    }
  } else {
    for (int i = 0; i < 8; ++i) {
      const float* p = row(position_of(r, tokens, t, section_of(r, j + i))) + j + i;
      x.c[i] = p[0], x.s[i] = p[half];
    }
  }
}

// The rotated elements.  No fused multiply-add: a key rounds to the same code
// wherever it is computed in plain fp32 products and sums.
__device__ __forceinline__ void turn(const Angles& x, bool interleaved, float (&a)[8], float (&b)[8]) {
#pragma clang fp contract(off)
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float(&y)[8] = i < 4 ? a : b;
      const float u = y[2 * (i % 4)], w = y[2 * (i % 4) + 1];
      y[2 * (i % 4)] = u * x.c[i] - w * x.s[i];
      y[2 * (i % 4) + 1] = w * x.c[i] + u * x.s[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = a[i], w = b[i];
      a[i] = u * x.c[i] - w * x.s[i];
      b[i] = w * x.c[i] + u * x.s[i];
    }
  }
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u; }

// The least 2^e, e in [kScaleMinExp, kScaleMaxExp], with amax <= 448 * 2^e.
__device__ __forceinline__ int scale_exp(float amax) {
  const uint32_t u = __float_as_uint(amax);
  // 448 = 1.75 * 2^8 (a subnormal amax has exponent field 0: the least scale)
  const int e = int(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kScaleMinExp), kScaleMaxExp);
}

// Four numbers to e4m3 codes, ties to even, beyond the range the largest.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  auto cut = [](float x) { return __builtin_amdgcn_fmed3f(x, -kE4m3Max, kE4m3Max); };
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(cut(a), cut(b), 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(cut(c), cut(d), r, true));
}
// Four codes moved to another scale; NaN codes stay (0x7f and 0xff hold no
// number that a factor below one could make finite, and the cut would).
__device__ __forceinline__ uint32_t rescaled4(uint32_t codes, float factor) {
  auto f = [&](auto hi) { return __builtin_amdgcn_cvt_pk_f32_fp8(int(codes), decltype(hi)::value); };
  const auto lo = f(std::false_type{}), hi = f(std::true_type{});
  uint32_t y = e4m3x4(lo[0] * factor, lo[1] * factor, hi[0] * factor, hi[1] * factor);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (((codes >> (8 * i)) & 0x7fu) == 0x7fu) y |= 0x7fu << (8 * i);
  return y;
}

// The largest of a and of b over the workgroup's 256 threads (kept in smem[8]).
__device__ __forceinline__ void block_max2(float& a, float& b, float* smem) {
  a = wave_max_f32(a), b = wave_max_f32(b);
  const int w = threadIdx.x / kWave;
  if (__lane_id() == 0) smem[w] = a, smem[4 + w] = b;
  __syncthreads();
  a = fmaxf(fmaxf(smem[0], smem[1]), fmaxf(smem[2], smem[3]));
  b = fmaxf(fmaxf(smem[4], smem[5]), fmaxf(smem[6], smem[7]));
}

// Stores go through byte merges where a 16-byte piece of the page also holds
// tokens that are not new: bytes of `fresh` where `mask` is set.
__device__ __forceinline__ uint32_t merge4(uint32_t old, uint32_t fresh, uint32_t mask) {
  return (old & ~mask) | (fresh & mask);
}
// Byte mask of the slots s0 .. s0 + 3 that lie in [lo, hi).
__device__ __forceinline__ uint32_t slots_mask(int s0, int lo, int hi) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (s0 + i >= lo && s0 + i < hi) m |= 0xffu << (8 * i);
  return m;
}

template <typename In, int D, int P>
__device__ void append_page(const AppendArgs& a, int b, const Seq& q, int nth, int h, char* smem) {
  constexpr int kLanes = D / 16;               // lanes of a key's row
  constexpr int kRows = kThreads / kLanes;     // rows the workgroup covers at once (keys)
  constexpr int kPasses = (P + kRows - 1) / kRows;
  constexpr int kQuads = (P / 4) * (D / 4);    // 4 x 4 squares of values
  constexpr int kSquares = (kQuads + kThreads - 1) / kThreads;
  constexpr int kSlots = kThreads / (D / 4) * 4;  // slots the workgroup covers at once (values)
  constexpr int kLd = P + 4;                   // bytes between channels of the turned values in LDS
  uint8_t* turned = reinterpret_cast<uint8_t*>(smem);            // [D][kLd]
  float* red = reinterpret_cast<float*>(smem + D * kLd);         // [8]
  uint32_t* bad = reinterpret_cast<uint32_t*>(smem + D * kLd + 32);  // [P]

  const int tid = threadIdx.x, Hkv = a.cache.kv_heads;
  const int place_lo = max(q.place0, 0), end = min(q.place0 + q.n, q.kv);
  const int entry = place_lo / P + nth;
  if (nth < 0 || entry * P >= end) return;  // (only where rows overlap, against the contract, in more than 2^31 pages)
  const int s0 = max(place_lo - entry * P, 0);   // slots [s0, s1) are new, [0, s0) held before
  const int s1 = min(end - entry * P, P);
  const int row0 = q.start + entry * P - q.place0;  // the call's row of slot 0

  for (int i = tid; i < P; i += kThreads) bad[i] = 0;

  // Positions and the page first, whatever waits for them behind the rows: a
  // small call is a chain of waits for memory (a step of 64 sequences took
  // 5.9 us with positions, angles and old scales each asked for when needed).
  // All rows are asked for before the first is used; a slot that is not new
  // reads a new one's row and leaves it (nothing branches around a load but
  // for whole passes without a new slot).
  auto row_of = [&](int slot) { return row0 + min(max(slot, s0), s1 - 1); };
  auto empty = [&](int lo, int n) { return lo >= s1 || lo + n <= s0; };
  const int lane = tid % kLanes, krow = tid / kLanes;  // of keys: lane of the row, row
  const Chunks ch = chunks_of(a.turn, lane);
  int position[kPasses];
#pragma unroll
  for (int i = 0; i < kPasses; ++i)
    position[i] = ch.turned && !empty(i * kRows, kRows) ? position_of(a.turn, a.batch.tokens, row_of(krow + i * kRows),
                                                                      section_of(a.turn, 8 * lane)) : 0;
  const int found = page_of(a.batch, a.cache.pages, b, entry), page = max(found, 0);
  // values: squares of 4 tokens x 4 channels, so that a token's four channels
  // are one load and a channel's four tokens one store
  Raw4<In> vr[kSquares][4];
#pragma unroll
  for (int i = 0; i < kSquares; ++i) {
    if (empty(i * kSlots, kSlots)) continue;
    const int sq = min(tid + i * kThreads, kQuads - 1), d = (sq % (D / 4)) * 4, t4 = (sq / (D / 4)) * 4;
#pragma unroll
    for (int r = 0; r < 4; ++r) vr[i][r].load(static_cast<const In*>(a.v) + row_of(t4 + r) * a.v_stride + h * D + d);
  }
  Raw8<In> kr[kPasses][2];
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    if (empty(i * kRows, kRows)) continue;
    const In* src = static_cast<const In*>(a.k) + row_of(krow + i * kRows) * a.k_stride + h * D;
    kr[i][0].load(src + ch.a), kr[i][1].load(src + ch.b);
  }
  float* const kscale = a.cache.k_scale + int64_t(page) * Hkv + h;
  float* const vscale = a.cache.v_scale + int64_t(page) * Hkv + h;
  const float ok = s0 > 0 ? *kscale : 0.f, ov = s0 > 0 ? *vscale : 0.f;
  Angles angle[kPasses];
#pragma unroll
  for (int i = 0; i < kPasses; ++i)
    if (ch.turned && !empty(i * kRows, kRows))
      angles(a.turn, a.batch.tokens, row_of(krow + i * kRows), lane, position[i], angle[i]);
  __syncthreads();  // `bad` is clear
  float kx[kPasses][2][8];
  float kmax = 0.f, vmax = 0.f;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    if (empty(i * kRows, kRows)) continue;
    const int slot = krow + i * kRows;
    kr[i][0].get(kx[i][0]), kr[i][1].get(kx[i][1]);
    if (ch.turned) turn(angle[i], a.turn.interleaved, kx[i][0], kx[i][1]);
    if (slot >= s0 && slot < s1) {
      bool nan = false;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = kx[i][e / 8][e % 8];
        if (finite(x)) kmax = fmaxf(kmax, fabsf(x));
        else nan = true;
      }
      if (nan) bad[slot] = 1;
    }
  }
  float vx[kSquares][4][4];
#pragma unroll
  for (int i = 0; i < kSquares; ++i) {
    const int sq = tid + i * kThreads, t4 = (sq / (D / 4)) * 4;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int slot = t4 + r;
      const bool in = !empty(i * kSlots, kSlots) && sq < kQuads && slot >= s0 && slot < s1;
      bool nan = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = in ? vr[i][r].get(e) : 0.f;
        if (!finite(x)) x = 0.f, nan = true;
        vmax = fmaxf(vmax, fabsf(x));
        vx[i][r][e] = x;
      }
      if (nan) bad[slot] = 1;
    }
  }
  block_max2(kmax, vmax, red);  // its barrier also covers `bad`
  if (found < 0) return;

  float ks = pow2(scale_exp(kmax)), vs = pow2(scale_exp(vmax)), kmove = 1.f, vmove = 1.f;
  if (s0 > 0) {
    if (ok < ks) kmove = ok / ks; else ks = ok;
    if (ov < vs) vmove = ov / vs; else vs = ov;
  }
  __syncthreads();  // the old scales are read by every thread
  if (tid == 0) *kscale = ks, *vscale = vs;
  const float kinv = 1.f / ks, vinv = 1.f / vs;

  uint8_t* const kpage = static_cast<uint8_t*>(a.cache.k) + (int64_t(page) * Hkv + h) * P * D;
  uint8_t* const vpage = static_cast<uint8_t*>(a.cache.v) + (int64_t(page) * Hkv + h) * P * D;
  if (kmove != 1.f)
    for (int i = tid; i < s0 * (D / 16); i += kThreads) {
      u32x4* p = reinterpret_cast<u32x4*>(kpage) + i;
      const u32x4 u = *p;
      *p = u32x4{rescaled4(u[0], kmove), rescaled4(u[1], kmove), rescaled4(u[2], kmove), rescaled4(u[3], kmove)};
    }
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int slot = krow + i * kRows;
    if (slot >= s0 && slot < s1) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float(&x)[8] = kx[i][c];
        u32x2 u{e4m3x4(x[0] * kinv, x[1] * kinv, x[2] * kinv, x[3] * kinv),
                e4m3x4(x[4] * kinv, x[5] * kinv, x[6] * kinv, x[7] * kinv)};
        if (bad[slot]) u = u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
        *reinterpret_cast<u32x2*>(kpage + slot * D + (c ? ch.b : ch.a)) = u;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kSquares; ++i) {
    const int sq = tid + i * kThreads, d = (sq % (D / 4)) * 4, t4 = (sq / (D / 4)) * 4;
    if (sq < kQuads) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<uint32_t*>(turned + (d + e) * kLd + t4) =
            e4m3x4(vx[i][0][e] * vinv, vx[i][1][e] * vinv, vx[i][2][e] * vinv, vx[i][3][e] * vinv);
    }
  }
  __syncthreads();
  // One or two new tokens: their bytes alone, without reading the pieces that
  // they lie in (a wait for memory less: 21.1 -> 18.6 us for a token each of 141
  // sequences and 16 heads).
  if (s1 - s0 <= 2 && vmove == 1.f) {
    for (int i = tid; i < D * (s1 - s0); i += kThreads) {
      const int d = i % D, slot = s0 + i / D;
      vpage[d * P + slot] = turned[d * kLd + slot];
    }
    return;
  }
  constexpr int kPieces = D * (P / 16);
  for (int i = tid; i < kPieces; i += kThreads) {
    const int d = i / (P / 16), t16 = (i % (P / 16)) * 16;
    const bool fresh = t16 < s1 && t16 + 16 > s0;
    if (!fresh && !(vmove != 1.f && t16 < s0)) continue;
    u32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = *reinterpret_cast<const uint32_t*>(turned + d * kLd + t16 + 4 * e);
    u32x4* const p = reinterpret_cast<u32x4*>(vpage + d * P + t16);
    if (t16 < s0 || t16 + 16 > s1) {
      const u32x4 old = *p;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int s = t16 + 4 * e;
        uint32_t was = old[e];
        if (vmove != 1.f) was = merge4(was, rescaled4(was, vmove), slots_mask(s, 0, s0));
        y[e] = merge4(was, y[e], slots_mask(s, s0, s1));
      }
    }
    *p = y;
  }
}

// Query rows: thread (lane of the row, head group, token); it keeps its angles
// over the heads it goes through, four of them asked for at once.
template <typename In, int D>
__device__ void rotate_queries(const AppendArgs& a, int unit, int heads_at_once) {
  constexpr int kLanes = D / 16, kBatch = 4;
  const int lane = threadIdx.x % kLanes, r = threadIdx.x / kLanes;
  const int per = kThreads / kLanes / heads_at_once;
  const int t = unit * per + r / heads_at_once;
  if (t >= a.batch.tokens) return;
  const Chunks ch = chunks_of(a.turn, lane);
  const In* src = static_cast<const In*>(a.q) + t * a.q_stride;
  uint16_t* dst = static_cast<uint16_t*>(a.q_out) + t * a.q_out_stride;
  const int position = ch.turned ? position_of(a.turn, a.batch.tokens, t, section_of(a.turn, 8 * lane)) : 0;
  Angles x;
  bool known = false;
  for (int h0 = r % heads_at_once; h0 < a.q_heads; h0 += kBatch * heads_at_once) {
    Raw8<In> raw[kBatch][2];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = min(h0 + i * heads_at_once, a.q_heads - 1);
      raw[i][0].load(src + h * D + ch.a), raw[i][1].load(src + h * D + ch.b);
    }
    if (!known && ch.turned) angles(a.turn, a.batch.tokens, t, lane, position, x);
    known = true;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = h0 + i * heads_at_once;
      float y[2][8];
      raw[i][0].get(y[0]), raw[i][1].get(y[1]);
      if (ch.turned) turn(x, a.turn.interleaved, y[0], y[1]);
      if (h < a.q_heads) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          bf16x8 z;
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = __bf16(y[c][e]);
          *reinterpret_cast<bf16x8*>(dst + h * D + (c ? ch.b : ch.a)) = z;
        }
      }
    }
  }
}

template <typename In, int D, int P>
__global__ __launch_bounds__(kThreads) void k_append(AppendArgs a, int page_groups, int heads_at_once) {
  __shared__ __align__(16) char smem[D * (P + 4) + 32 + 4 * P];
  const int id = blockIdx.x;
  if (id >= page_groups) {
    rotate_queries<In, D>(a, id - page_groups, heads_at_once);
    return;
  }
  auto touched = [](const Seq& q) {
    const int lo = max(q.place0, 0), hi = min(q.place0 + q.n, q.kv);
    return hi > lo ? (hi - 1) / P - lo / P + 1 : 0;
  };
  const Found f = find_item(a.batch, id / a.cache.kv_heads, touched);
  if (f.seq < 0) return;
  append_page<In, D, P>(a, f.seq, f.s, f.local, id % a.cache.kv_heads, smem);
}

template <typename In, int D>
hipError_t launch(const AppendArgs& a, int groups, int units, int heads_at_once, hipStream_t s) {
  const dim3 grid(groups + units), block(kThreads);
  switch (a.cache.page_size) {
    case 16: hipLaunchKernelGGL((k_append<In, D, 16>), grid, block, 0, s, a, groups, heads_at_once); break;
    case 32: hipLaunchKernelGGL((k_append<In, D, 32>), grid, block, 0, s, a, groups, heads_at_once); break;
    case 64: hipLaunchKernelGGL((k_append<In, D, 64>), grid, block, 0, s, a, groups, heads_at_once); break;
    default: hipLaunchKernelGGL((k_append<In, D, 128>), grid, block, 0, s, a, groups, heads_at_once); break;
  }
  return hipGetLastError();
}

}  // namespace

namespace {

struct Grid {
  int64_t groups, units;  // workgroups of pages, and of queries
  int heads_at_once;
};
Grid append_grid(const wz_cache& c, const wz_ragged& r, int q_heads) {
  const int P = c.page_size;
  Grid g{};
  // pages that receive tokens: at most one a token, (n + P - 2) / P + 1 a
  // sequence, and tokens / P and two more a sequence together
  if (r.max_tokens > 0)
    g.groups = c.kv_heads * std::min({int64_t(r.tokens), int64_t(r.batch) * ((r.max_tokens + P - 2) / P + 1),
                                      int64_t(r.tokens / P) + 2 * int64_t(r.batch)});
  g.heads_at_once = 1;  // a thread has four heads or more where there are as many
  while (g.heads_at_once < 8 && 4 * g.heads_at_once < q_heads) g.heads_at_once *= 2;
  const int per = kThreads / (c.head_dim / 16) / g.heads_at_once;
  g.units = q_heads ? (int64_t(r.tokens) + per - 1) / per : 0;
  return g;
}

}  // namespace

int64_t append_groups(const wz_cache& c, const wz_ragged& r, int q_heads) {
  const Grid g = append_grid(c, r, q_heads);
  return g.groups + g.units;
}

hipError_t launch_append(const AppendArgs& a, int in_dtype, hipStream_t s) {
  const Grid g = append_grid(a.cache, a.batch, a.q_heads);
  if (g.groups + g.units == 0) return hipSuccess;
  const int groups = int(g.groups), units = int(g.units);
  const bool bf = in_dtype == WZ_BF16;
  if (a.cache.head_dim == 128)
    return bf ? launch<uint16_t, 128>(a, groups, units, g.heads_at_once, s)
              : launch<float, 128>(a, groups, units, g.heads_at_once, s);
  return bf ? launch<uint16_t, 64>(a, groups, units, g.heads_at_once, s)
            : launch<float, 64>(a, groups, units, g.heads_at_once, s);
}

}  // namespace wz
