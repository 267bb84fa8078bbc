// Linear attention with a decay for each head, a chunk of 64 tokens at a time
// (wz_decay_attention).
//
// With l the head's decay, S the state that a chunk of n tokens begins with, and
// i, t < n its tokens,
//   out_i = scale (l^(i+1) q_i S + sum_{t <= i} l^(i-t) (q_i . k_t) v_t)
//   S'    = l^n S + sum_t k_t (l^(n-1-t) v_t)^T
// which are products of matrices.  The state stays in the accumulators of the
// last product, one wave to 32 columns of it, from chunk to chunk: as the left
// operand of q S it needs no other place, since the order of a sum over the
// rows of S may be that of the accumulator's registers (q and k are laid out in
// that order once, as they are stored in LDS).
//
// Factors that are not bf16 already are taken apart: the state's sums take the
// decayed values in three parts, which is all of their 24 bits; the outputs, which
// are rounded to bf16 themselves, take the state and the decayed scores in two.
#include "wz_decay.h"

namespace wz {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kChunk = 64;

__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// The upper halves of two numbers: both cut to bf16.
__device__ __forceinline__ uint32_t upper(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);
}
// 2^x; below fp32's normal numbers zero.
__device__ __forceinline__ float power(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rest(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ uint32_t pair(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{__bf16(lo), __bf16(hi)});
}

// Where a sequence's segment begins: its state in the workspace, in the order of
// the accumulators ([wave][rows of 32][16 rows of those in four][lane], four
// numbers each).
template <int D>
__device__ __forceinline__ f32x4* begins(const DecayArgs& p, int b, int seg, int h, int wave) {
  return reinterpret_cast<f32x4*>(p.part + ((int64_t(b) * p.segments + seg) * p.states.heads + h) * (D * D)) +
         wave * (D / 32) * 4 * kWave + __lane_id();
}

// OUT: outputs and the last state; otherwise what a segment adds to the state.
template <int D, bool OUT>
__global__ __launch_bounds__(2 * D, 2) void k_decay_prompt(DecayArgs p) {
  constexpr int W = D / 32, NA = D / 32, kUnits = D / 8;  // waves; tiles of the state's rows; 16-byte units of a row
  // (scores are written where the keys lay, once every wave is done with those)
  constexpr int kScores = 2 * kChunk * kChunk;
  __shared__ __align__(256) uint16_t lds[OUT ? 3 * kChunk * D + (kChunk * D > kScores ? kChunk * D : kScores) : 2 * kChunk * D];
  __shared__ __align__(16) float weight[kChunk];
  __shared__ uint32_t odd[2][2];  // tokens with a number that is none, of this chunk and of the next
  // [D][64 tokens] keys, values; [64][D] queries, keys, in the order of the accumulators' rows; [2 parts][64][64
  // tokens] scores: bytes from the beginning
  constexpr uint32_t kt = 0, vt = 2 * kChunk * D, qs = 2 * vt, ks = 3 * vt, sc = ks;
  constexpr uint32_t kRow = 2 * D, kCol = 2 * kChunk;  // bytes of a row
  auto at16 = [&](uint32_t to) -> u32x4& { return *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(lds) + to); };
  auto at8 = [&](uint32_t to) -> u32x2& { return *reinterpret_cast<u32x2*>(reinterpret_cast<char*>(lds) + to); };
  auto at2 = [&](uint32_t to) -> uint16_t& { return *reinterpret_cast<uint16_t*>(reinterpret_cast<char*>(lds) + to); };

  const int lane = __lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), c = lane & 31, g = lane >> 5;
  const int h = blockIdx.x % p.states.heads, rest_id = blockIdx.x / p.states.heads;
  const int segs = OUT ? p.segments : p.segments - 1;
  const int seg = rest_id % segs, b = rest_id / segs;
  const Seq s = sequence(p.batch, b);
  const int first = p.segments > 1 ? seg * p.segment : 0;
  const int last = p.segments > 1 ? min(s.n, first + p.segment) : s.n;
  // (a segment that is its sequence's last adds to no other's beginning)
  if (first >= s.n || (!OUT && last >= s.n)) return;
  const int slot = p.slot[b];
  const bool kept = uint32_t(slot) < uint32_t(p.states.slots);
  float* const state = p.states.state + (int64_t(kept ? slot : 0) * p.states.heads + h) * (D * D) + wave * 32 + c;
  float ld = log2_decay(p, h);
  const int b0 = wave * 32;

  f32x16 S[NA] = {};
  if constexpr (OUT) {
    if (p.segments > 1) {
      const f32x4* from = begins<D>(p, b, seg, h, wave);
#pragma unroll
      for (int i = 0; i < NA * 4; ++i) {
        const f32x4 x = from[i * kWave];
#pragma unroll
        for (int e = 0; e < 4; ++e) S[i / 4][i % 4 * 4 + e] = x[e];
      }
    } else if (kept && s.place0 > 0) {
#pragma unroll
      for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) S[a][r] = state[(32 * a + 8 * (r / 4) + 4 * g + r % 4) * D];
    }
  }

  // A thread moves four tokens' 16 bytes of queries, keys and values.
  int unit = threadIdx.x % kUnits, quad = threadIdx.x / kUnits;
  const int kh = h / p.group;
  const uint16_t* const qp = static_cast<const uint16_t*>(p.q) + s.start * p.q_stride + h * D + 8 * unit;
  const uint16_t* const kp = static_cast<const uint16_t*>(p.k) + s.start * p.k_stride + kh * D + 8 * unit;
  const uint16_t* const vp = static_cast<const uint16_t*>(p.v) + s.start * p.v_stride + kh * D + 8 * unit;
  u32x4 nq[4], nk[4], nv[4];
  auto fetch = [&](int t0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = min(t0 + 4 * quad + i, last - 1);
      if constexpr (OUT) nq[i] = *reinterpret_cast<const u32x4*>(qp + t * p.q_stride);
      nk[i] = *reinterpret_cast<const u32x4*>(kp + t * p.k_stride);
      nv[i] = *reinterpret_cast<const u32x4*>(vp + t * p.v_stride);
    }
  };
  // The 16-byte units of a row are exchanged by the row's number, so that 16 lanes
  // that read one unit of 16 rows hit all banks, and writes of four tokens half of
  // them.  The number is the unit's xor some bits of the row's: a lane's reads differ by
  // an xor with constants.
  auto row_x = [](int row) { return kUnits == 16 ? row & 15 : row >> 1 & 7; };
  auto col_x = [](int row) { return (row >> 1 ^ row >> 4) & 7; };
  auto row_at = [&](uint32_t base, int row, int u) { return base + row * kRow + 16 * (u ^ row_x(row)); };
  auto col_at = [&](uint32_t base, int row, int u) { return base + row * kCol + 16 * (u ^ col_x(row)); };
  // this lane's unit g of rows c (the others: rows 32 i + c, units 2 k + g)
  uint32_t my_row = row_at(0, c, g), my_col = col_at(0, c, g), my_sc = c * kCol + 16 * (g ^ (c >> 1 & 7));
  auto read_row = [&](uint32_t base, int i, int k) -> u32x4 { return at16(base + 32 * i * kRow + (my_row ^ 32 * k)); };
  auto read_col = [&](uint32_t base, int i, int k) -> u32x4 { return at16(base + 32 * i * kCol + (my_col ^ 32 * (k ^ i))); };
  auto read_sc = [&](int part, int i, int k) -> u32x4 { return at16(sc + (64 * part + 32 * i) * kCol + (my_sc ^ 32 * k)); };
  auto store_rows = [&](uint32_t base, const u32x4 (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int half = 0; half < 2; ++half)
        at8(row_at(base, 4 * quad + i, unit / 2 * 2 + half) + 8 * (unit & 1)) =
            u32x2{x[i][2 * half], x[i][2 * half + 1]};
  };
  auto store_columns = [&](uint32_t base, const u32x4 (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t pick = e % 2 ? 0x07060302 : 0x05040100;
      at8(col_at(base, 8 * unit + e, quad / 2) + 8 * (quad & 1)) =
          u32x2{__builtin_amdgcn_perm(x[1][e / 2], x[0][e / 2], pick), __builtin_amdgcn_perm(x[3][e / 2], x[2][e / 2], pick)};
    }
  };

  if (threadIdx.x < 4) odd[threadIdx.x / 2][threadIdx.x % 2] = 0;
  __syncthreads();
  fetch(first);
  int parity = 0;
  for (int t0 = first; t0 < last; t0 += kChunk, parity ^= 1) {
    const int len = min(kChunk, last - t0);
    asm volatile("" : "+v"(unit), "+v"(quad));
    // a key or a value that is no number, by its exponent
    uint32_t strange = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = 4 * quad + i < len;
      typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
      u16x2 top = {};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        nk[i][e] = in ? nk[i][e] : 0u, nv[i][e] = in ? nv[i][e] : 0u;
        if constexpr (OUT) nq[i][e] = in ? nq[i][e] : 0u;
        top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, nk[i][e] & 0x7fff7fffu));
        top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, nv[i][e] & 0x7fff7fffu));
      }
      strange |= top[0] >= 0x7f80 || top[1] >= 0x7f80 ? 1u << i : 0u;
    }
    if (strange) atomicOr(&odd[parity][quad / 8], strange << (4 * quad & 31));
    auto weigh = [&](int end) {  // a token's decay up to the one before `end`
      if (threadIdx.x < kChunk) weight[threadIdx.x] = power(float(max(end - 1 - int(threadIdx.x), 0)) * ld);
    };
    if (t0 == first || len < kChunk) weigh(len);
    store_columns(kt, nk);
    store_columns(vt, nv);
    if constexpr (OUT) {
      store_rows(qs, nq);
      store_rows(ks, nk);
    }
    __syncthreads();
    if (threadIdx.x < 2) odd[parity ^ 1][threadIdx.x] = 0;  // (read by none before the next chunk's barrier)
    const uint64_t marked = uint64_t(__builtin_amdgcn_readfirstlane(odd[parity][1])) << 32 |
                            uint32_t(__builtin_amdgcn_readfirstlane(odd[parity][0]));
    if (!marked && t0 + kChunk < last) fetch(t0 + kChunk);
    uint16_t* const out = OUT ? static_cast<uint16_t*>(p.out) + (s.start + t0) * p.out_stride + h * D + b0 : nullptr;
    // In a product with zeros what is no number would reach rows that do not see it:
    // a chunk is worked on in pieces, a token with such a number and those between two
    // of them, the others' keys and values being zeros.  (All but always: one piece.)
    for (int u0 = 0, u1; u0 < len; u0 = u1) {
    // (what is worked out from these is not worth a register from chunk to chunk)
    int row = c, four = 4 * g;
    asm volatile("" : "+v"(my_row), "+v"(my_col), "+v"(my_sc), "+v"(ld), "+v"(row), "+v"(four));
    const uint64_t ahead = marked >> u0;
    u1 = ahead & 1 ? u0 + 1 : ahead ? u0 + __builtin_ctzll(ahead) : len;
    if (marked) {
      __syncthreads();
      weigh(u1);
      if constexpr (OUT) store_rows(ks, nk);  // (where the last piece's scores were)
      __syncthreads();
    }
    auto piece = [&](int k, u32x4& x) {
      if (marked) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = 16 * k + 2 * four + 2 * e;
          x[e] &= (t >= u0 && t < u1 ? 0xffffu : 0u) | (t + 1 >= u0 && t + 1 < u1 ? 0xffff0000u : 0u);
        }
      }
    };
    u32x4 vf[4];
    auto read_values = [&] {
#pragma unroll
      for (int k = 0; k < 4; ++k) vf[k] = read_col(vt, wave, k), piece(k, vf[k]);
    };
    if constexpr (OUT) {
      // Scores of 32 x 32 (tokens down, queries across), three of the chunk's four: (0, 0), (32, 32), and (0, 32).
      constexpr int kMine = (3 + W - 1) / W;
      f32x16 X[kMine] = {};
#pragma unroll
      for (int m = 0; m < kMine; ++m) {
        const int tile = wave + m * W;
        if (tile < 3) {
          const int kr = tile == 1, qr = tile != 0;
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            X[m] = mfma(read_row(ks, kr, k), read_row(qs, qr, k), X[m]);
            if (k % 2) __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int m = 0; m < kMine; ++m) {
        const int tile = wave + m * W;
        if (tile < 3) {
          const int kr = tile == 1, qr = tile != 0;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int t = 8 * q + four + e, gap = 32 * (qr - kr) + row - t;
              const float x = X[m][4 * q + e] * power(float(max(gap, 0)) * ld);
              y[e] = min(gap, 32 * kr + t - u0) >= 0 ? x : 0.f;
            }
            const uint32_t to = sc + 32 * qr * kCol + ((my_sc ^ 4 * four) ^ 16 * (4 * kr + q)) + 2 * four;
            at8(to) = u32x2{upper(y[0], y[1]), upper(y[2], y[3])};
            at8(to + 64 * kCol) = u32x2{pair(rest(y[0]), rest(y[1])), pair(rest(y[2]), rest(y[3]))};
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      f32x16 O[2] = {};
#pragma unroll
      for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          u32x4 hi, lo;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = S[a][8 * kk + 2 * e], y = S[a][8 * kk + 2 * e + 1];
            hi[e] = upper(x, y), lo[e] = pair(rest(x), rest(y));
          }
          const u32x4 q0 = read_row(qs, 0, 2 * a + kk), q1 = read_row(qs, 1, 2 * a + kk);
          O[0] = mfma(hi, q0, O[0]);
          O[1] = mfma(hi, q1, O[1]);
          O[0] = mfma(lo, q0, O[0]);
          O[1] = mfma(lo, q1, O[1]);
          if (kk) __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float f = power(float(max(32 * i + row + 1 - u0, 0)) * ld);
#pragma unroll
        for (int r = 0; r < 16; ++r) O[i][r] *= f;
      }
      __syncthreads();
      read_values();
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          if (k < 2) O[0] = mfma(vf[k], read_sc(part, 0, k), O[0]);
          O[1] = mfma(vf[k], read_sc(part, 1, k), O[1]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (32 * i + row >= u0 && 32 * i + row < u1) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *reinterpret_cast<u32x2*>(out + (32 * i + row) * p.out_stride + 8 * q + four) =
                u32x2{pair(O[i][4 * q] * p.scale, O[i][4 * q + 1] * p.scale),
                      pair(O[i][4 * q + 2] * p.scale, O[i][4 * q + 3] * p.scale)};
        }
    } else {
      read_values();
    }
    const float fade = power(float(u1 - u0) * ld);
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int r = 0; r < 16; ++r) S[a][r] *= fade;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      u32x4 part[3];
      f32x4 w[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) w[e] = *reinterpret_cast<const f32x4*>(weight + 16 * k + 2 * four + 4 * e);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = bf16_lo(vf[k][e]) * w[e / 2][e % 2 * 2], y = bf16_hi(vf[k][e]) * w[e / 2][e % 2 * 2 + 1];
        const float x1 = rest(x), y1 = rest(y);
        part[0][e] = upper(x, y), part[1][e] = upper(x1, y1), part[2][e] = upper(rest(x1), rest(y1));
      }
      u32x4 kf[NA];
#pragma unroll
      for (int a = 0; a < NA; ++a) kf[a] = read_col(kt, a, k), piece(k, kf[a]);
#pragma unroll
      for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int a = 0; a < NA; ++a) S[a] = mfma(kf[a], part[i], S[a]);
      __builtin_amdgcn_sched_barrier(0);
    }
    }
    __syncthreads();
    if (marked && t0 + kChunk < last) {
      fetch(t0 + kChunk);
      weigh(kChunk);
    }
  }

  if constexpr (!OUT) {
    f32x4* to = begins<D>(p, b, seg + 1, h, wave);
#pragma unroll
    for (int i = 0; i < NA * 4; ++i)
      to[i * kWave] = f32x4{S[i / 4][i % 4 * 4], S[i / 4][i % 4 * 4 + 1], S[i / 4][i % 4 * 4 + 2], S[i / 4][i % 4 * 4 + 3]};
  } else if (kept && last == s.n) {
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int r = 0; r < 16; ++r) state[(32 * a + 8 * (r / 4) + 4 * g + r % 4) * D] = S[a][r];
  }
}

// The state that each segment of a sequence begins with, from what those before
// it add: four numbers a thread.
template <int D>
__global__ __launch_bounds__(256) void k_decay_join(DecayArgs p) {
  constexpr int kParts = D * D / 4 / 256;  // workgroups of a sequence and head
  const int part = blockIdx.x % kParts, h = blockIdx.x / kParts % p.states.heads, b = blockIdx.x / kParts / p.states.heads;
  const Seq s = sequence(p.batch, b);
  if (s.n <= 0) return;
  const int slot = p.slot[b], lane = __lane_id();
  const int at = (part * 256 + threadIdx.x) / kWave, wave = at / (D / 8), i = at % (D / 8);  // in the accumulators' order
  f32x4 S = {};
  if (uint32_t(slot) < uint32_t(p.states.slots) && s.place0 > 0) {
    const float* state = p.states.state + (int64_t(slot) * p.states.heads + h) * (D * D) + wave * 32 + (lane & 31);
#pragma unroll
    for (int e = 0; e < 4; ++e) S[e] = state[(32 * (i / 4) + 8 * (i % 4) + 4 * (lane >> 5) + e) * D];
  }
  const float fade = power(float(p.segment) * log2_decay(p, h));
  const int segs = (s.n + p.segment - 1) / p.segment;
  f32x4* to = begins<D>(p, b, 0, h, wave) + i * kWave;
  const int64_t next = int64_t(p.states.heads) * (D * D / 4);
  for (int j = 0; j < segs; ++j, to += next) {
    if (j > 0) {
      const f32x4 x = *to;
#pragma unroll
      for (int e = 0; e < 4; ++e) S[e] = fmaf(S[e], fade, x[e]);
    }
    *to = S;
  }
}

template <int D>
hipError_t prompt(const DecayArgs& p, hipStream_t s) {
  const uint32_t pairs = uint32_t(p.batch.batch) * p.states.heads;
  if (p.segments > 1) {
    hipLaunchKernelGGL((k_decay_prompt<D, false>), dim3(pairs * (p.segments - 1)), dim3(2 * D), 0, s, p);
    hipLaunchKernelGGL((k_decay_join<D>), dim3(pairs * (D * D / 1024)), dim3(256), 0, s, p);
  }
  hipLaunchKernelGGL((k_decay_prompt<D, true>), dim3(pairs * p.segments), dim3(2 * D), 0, s, p);
  return hipGetLastError();
}

}  // namespace

// A workgroup to a sequence and head, or to a segment of it where those are fewer
// than the CUs hold.
DecayPlan decay_plan(const wz_states& z, const wz_ragged& r) {
  DecayPlan p{};
  p.token = r.max_tokens <= 16;
  p.segments = 1, p.segment = r.max_tokens;
  if (p.token) return p;
  const int64_t pairs = int64_t(r.batch) * z.heads, room = 2 * kCUs;
  const int chunks = (r.max_tokens + kChunk - 1) / kChunk;
  const int64_t want = std::min<int64_t>(room / pairs, chunks / 2);
  if (want > 1) {
    p.segment = int((chunks + want - 1) / want) * kChunk;
    p.segments = (r.max_tokens + p.segment - 1) / p.segment;
  }
  if (p.segments > 1) p.bytes = size_t(pairs) * p.segments * z.head_dim * z.head_dim * 4;
  return p;
}

hipError_t launch_decay_prompt(const DecayArgs& p, hipStream_t s) {
  return p.states.head_dim == 128 ? prompt<128>(p, s) : prompt<64>(p, s);
}

}  // namespace wz
