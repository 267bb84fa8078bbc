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
// (With one part less each, eight long prompts took 2 to 9 % less.)
//
// Measured (28 heads of 128 elements): a prompt of 1286 tokens 35 to 40 us, eight of 3531 to
// 9459 541 to 575 us, 0.17 PFLOP/s of what the formula asks for.  Their operations and bytes
// would allow 5 and 291 us.  A chunk takes 5.4 us where a CU has one workgroup, and 8.4 where
// it has two: scores, q S, scores times values and the state one after the other, with four
// barriers.  No pipe is full (vector ALU 36 % of the cycles, MFMA 36 %, LDS 28 %); registers
// allow two waves a SIMD to overlap them.
#include <cmath>

#include "wz_decay.h"

namespace wz {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kChunk = 64;
constexpr float kRaised = 16.f;  // log2 of what a state is raised by at most
// For outputs a state is kept this much lower, so that raised it is what it stands for at most, and q S, which is
// formed from it, passes fp32 no sooner than the formula's.
constexpr float kLower = 0x1p-16f, kHigher = 0x1p16f;

__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}
__device__ __forceinline__ uint32_t pair(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, bf16x2{__bf16(lo), __bf16(hi)});
}
// c and the products of two pairs of bf16.
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), c, false);
}
// Two numbers cut to bf16 (their upper halves), and what that leaves of them: a
// product with -1 and a sum in one instruction.  The constants have to lie in
// vector registers.
struct Cut {
  uint32_t low, high;  // (-1, 0) and (0, -1)
  __device__ __forceinline__ uint32_t operator()(float& x, float& y) const {
    const uint32_t u = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302);
    x = dot2(u, low, x), y = dot2(u, high, y);
    return u;
  }
};
// 2^x; below fp32's normal numbers zero.
__device__ __forceinline__ float power(float x) { return __builtin_amdgcn_exp2f(x); }

// A state in the workspace, in the order of the accumulators ([wave][rows of 32]
// [16 rows of those in four][lane], four numbers each).
__device__ __forceinline__ float* stored(const DecayArgs& p, int kind, int run, int h) {
  return p.part + ((int64_t(kind) * p.runs + run) * p.states.heads + h) * (p.states.head_dim * p.states.head_dim);
}
constexpr int kBegins = 0;  // of a run's first sequence, if that goes on from another run: what the run before this
                            // one adds (to zeros, or to kFirst), and then, if the sums are joined, what it begins with
constexpr int kFirst = 1;   // what a run's last sequence has before the call, if that begins in the run and goes on

// Chunks from one sequence to the next: a run's are [lo, hi) of all.
__device__ __forceinline__ int chunks_of(const Seq& s) { return (s.n + kChunk - 1) / kChunk; }
struct Run {
  int seq, at;  // its first chunk's sequence, and the chunk's number there
  int chunks;
  int all, runs;  // of the call: chunks, and runs that have any
};
// The first of `all` chunks that a run has: the first runs have one more than the others.
__device__ __forceinline__ int first_of(int run, int all, int runs) {
  const int each = uint32_t(all) / uint32_t(runs);
  return run * each + min(run, all - each * runs);
}
// LAST: of the run, what belongs to its last sequence.
template <bool LAST>
__device__ __forceinline__ Run run_of(const DecayArgs& p, int run) {
  if (p.runs == 0) return Run{run, 0, chunks_of(sequence(p.batch, run)), 0, 0};  // a sequence each
  const int lane = __lane_id();
  int all = 0, mine = 0, incl = 0;  // (of 64 sequences at a time: this lane's, and those up to it)
  for (int b = 0; b < p.batch.batch; b += kWave) {
    mine = b + lane < p.batch.batch ? chunks_of(sequence(p.batch, b + lane)) : 0;
    incl = wave_incl_scan_i32(mine);
    all += __builtin_amdgcn_readlane(incl, kWave - 1);
  }
  // (fewer chunks than the bounds promise: a run each, and none behind, since what a sequence has before a run is
  // handed on by the run before it)
  const int runs = min(p.runs, all);
  if (run >= runs) return Run{};
  const int lo = first_of(run, all, runs), hi = first_of(run + 1, all, runs);
  const int item = LAST ? hi - 1 : lo;
  int seq, at;
  if (p.batch.batch <= kWave) {
    seq = __builtin_ctzll(__ballot(incl > item));
    at = item - __builtin_amdgcn_readlane(incl, seq) + __builtin_amdgcn_readlane(mine, seq);
  } else {
    const Found f = find_item(p.batch, item, [](const Seq& s) { return chunks_of(s); });
    if (f.seq < 0) return Run{};  // (rows that overlap against the contract, past 32 bits)
    seq = f.seq, at = f.local;
  }
  if (!LAST) return Run{seq, at, hi - lo, all, runs};
  const int first = max(at - (hi - 1 - lo), 0);
  return Run{seq, first, at - first + 1, all, runs};
}

// A workgroup goes through a run of chunks.  OUT: outputs, and the sequences' last
// states.  Otherwise, where the run's last sequence goes on in the next run, what
// its chunks here add to the state.
template <int D, bool OUT>
__global__ __launch_bounds__(2 * D, 2) void k_decay_prompt(DecayArgs p) {
  constexpr int W = D / 32, NA = D / 32, kUnits = D / 8;  // waves; tiles of the state's rows; 16-byte units of a row
  // [D][64 tokens] keys, values; [64][D] queries, keys, in the order of the accumulators' rows; [2 parts][64][64
  // tokens] scores, where the keys lay, once every wave is done with those
  constexpr int kt = 0, vt = 2 * kChunk * D, qs = 2 * vt, ks = 3 * vt, sc = ks;
  constexpr int kRow = 2 * D, kCol = 2 * kChunk;  // bytes of a row
  __shared__ __align__(256) char lds[OUT ? ks + (vt > 2 * 64 * kCol ? vt : 2 * 64 * kCol) : qs];
  __shared__ __align__(16) float weight[kChunk];
  __shared__ int strange[OUT ? D : 1];  // of each element of the values, the first token where it is no number

  const int lane = __lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c = lane & 31, g = lane >> 5;
  // Workgroups go to the XCDs in turn: heads that share a key head to the same
  // one, whose L2 they read it from.
  const int x = blockIdx.x % kXcds, y = blockIdx.x / kXcds, kv_heads = p.states.heads / p.group;
  const int runs = p.runs ? p.runs : p.batch.batch, set = y / p.group * kXcds + x;
  if (set >= runs * kv_heads) return;
  const int kh = set % kv_heads, h = kh * p.group + y % p.group, run = set / kv_heads;
  const Run all = run_of<!OUT>(p, run);
  int goes_on = 0;
  float ld = log2_decay(p, h);
  const int b0 = wave * 32;

  Seq s;
  int last;  // behind the last token of the sequence in this run
  // A thread moves four tokens' 16 bytes of queries, keys and values.  Tokens behind
  // the last one lie behind the buffer's end and read as zeros.
  int unit = threadIdx.x % kUnits, quad = threadIdx.x / kUnits;
  u32x4 nq[4], nk[4], nv[4];
  auto get = [&](const void* base, int64_t stride, int head, int t0, u32x4 (&to)[4]) {
    const int rows = min(kChunk, last - t0);
    const auto r = make_rsrc_uniform(static_cast<const uint16_t*>(base) + (s.start + t0) * stride + head * D,
                                     uint32_t((rows - 1) * int(stride) + D) * 2);
    int at = 4 * quad * int(2 * stride) + 16 * unit;
#pragma unroll
    for (int i = 0; i < 4; ++i, at += int(2 * stride)) to[i] = buf_load_u32x4(r, at);
  };
  auto fetch = [&](int t0) {
    get(p.k, p.k_stride, kh, t0, nk);
    get(p.v, p.v_stride, kh, t0, nv);
    if constexpr (OUT) get(p.q, p.q_stride, h, t0, nq);
  };
  // (barriers order LDS alone: the next chunk's loads stay under way)
  //
  // The 16-byte units of a row are exchanged by the row's number, so that 16 lanes
  // that read one unit of 16 rows hit all banks, and writes of four tokens half of
  // them.  A unit's place is its number xor some bits of the row's: a lane's reads
  // differ by an xor with constants.
  auto row_x = [](int row) { return kUnits == 16 ? row & 15 : row >> 1 & 7; };
  auto col_x = [](int row) { return (row >> 1 ^ row >> 4) & 7; };
  // this lane's unit g of rows c (its others: rows 32 i + c, units 2 k + g)
  int my_row = c * kRow + 16 * (g ^ row_x(c)), my_col = c * kCol + 16 * (g ^ col_x(c));
  int my_sc = c * kCol + 16 * (g ^ (c >> 1 & 7));
  auto read = [&](int to, int more) { return *reinterpret_cast<const u32x4*>(lds + to + more); };
  auto read_row = [&](int base, int i, int k) { return read(my_row ^ 32 * k, base + 32 * i * kRow); };
  auto read_col = [&](int base, int i, int k) { return read(my_col ^ 32 * (k ^ i), base + 32 * i * kCol); };
  auto read_sc = [&](int part, int i, int k) { return read(my_sc ^ 32 * k, sc + (64 * part + 32 * i) * kCol); };
  auto write8 = [&](int to, int more, uint32_t lo, uint32_t hi) {
    *reinterpret_cast<u32x2*>(lds + to + more) = u32x2{lo, hi};
  };
  auto store_rows = [&](int base, const u32x4 (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * quad + i, to = row * kRow + 16 * ((unit & ~1) ^ row_x(row)) + 8 * (unit & 1);
      write8(to, base, v[i][0], v[i][1]);
      write8(to ^ 16, base, v[i][2], v[i][3]);
    }
  };
  auto store_columns = [&](int base, const u32x4 (&v)[4]) {
    const int to = 8 * unit * kCol + 16 * (quad / 2 ^ col_x(8 * unit)) + 8 * (quad & 1);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t pick = e % 2 ? 0x07060302 : 0x05040100;
      write8(to ^ 16 * (e >> 1), base + e * kCol, __builtin_amdgcn_perm(v[1][e / 2], v[0][e / 2], pick),
             __builtin_amdgcn_perm(v[3][e / 2], v[2][e / 2], pick));
    }
  };
  Cut cut{0x0000bf80u, 0xbf800000u};
  uint32_t zero = 0;
  asm volatile("" : "+v"(cut.low), "+v"(cut.high), "+v"(zero));

  // the decays from a score's token to its query, and the scale
  constexpr int kMine = OUT ? (3 + W - 1) / W : 1;  // of the three tiles of scores
  f32x16 by_gap[kMine];
  if constexpr (OUT) {
#pragma unroll
    for (int m = 0; m < kMine; ++m)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        by_gap[m][r] =
            power(float(max((wave + m * W == 2 ? 32 : 0) + c - 4 * g - 8 * (r / 4) - r % 4, 0)) * ld) * p.scale;
  }
  int b = all.seq, at = all.at, left = all.chunks;
  while (left > 0 && b < p.batch.batch) {
    s = sequence(p.batch, b);
    const int chunks = min(chunks_of(s) - at, left), first = at * kChunk;
    if (OUT && chunks <= 0) {  // (a sequence without tokens)
      ++b, at = 0;
      continue;
    }
    left -= chunks;
    last = min(s.n, first + chunks * kChunk);
    const bool on = last < s.n;  // in the next run
    if (!OUT && !on) break;
    const int slot = p.slot[b];
    const bool kept = uint32_t(slot) < uint32_t(p.states.slots);
    const auto state =
        make_rsrc_uniform(p.states.state + (int64_t(kept ? slot : 0) * p.states.heads + h) * (D * D), D * D * 4);
    auto row_of = [](int a, int r) { return 4 * D * (32 * a + 8 * (r / 4) + r % 4); };  // bytes from the lane's first
    // this lane's element of a state's first row of four, and its first four in the accumulators' order
    int in_state = 4 * (4 * g * D + wave * 32 + c), in_order = 16 * (wave * NA * 4 * kWave + lane);
    asm volatile("" : "+v"(in_state), "+v"(in_order));
    f32x16 S[NA] = {};
    auto from = [&](const float* base, float f) {  // (added, times f)
      const auto r = make_rsrc_uniform(base, D * D * 4);
      f32x4 v[NA * 4];
#pragma unroll
      for (int i = 0; i < NA * 4; ++i)
        v[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, in_order, i * 16 * kWave, 0));
#pragma unroll
      for (int i = 0; i < NA * 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[i / 4][i % 4 * 4 + e] = fmaf(v[i][e], f, S[i / 4][i % 4 * 4 + e]);
    };
    auto into = [&](float* base) {
      const auto r = make_rsrc_uniform(base, D * D * 4);
#pragma unroll
      for (int i = 0; i < NA * 4; ++i) {
        const f32x16& x = S[i / 4];
        const f32x4 v = {x[i % 4 * 4], x[i % 4 * 4 + 1], x[i % 4 * 4 + 2], x[i % 4 * 4 + 3]};
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, in_order, i * 16 * kWave, 0);
      }
    };
    if (OUT && first > 0 && !p.join) {  // what the sequence's runs before this one add, from the last one on
      const int here = first_of(run, all.all, all.runs), begins = here - first / kChunk;
      for (int r = run; r > 0; --r) {
        const int before = first_of(r, all.all, all.runs);
        if (before <= begins) break;
        from(stored(p, kBegins, r, h), power(float((here - before) * kChunk) * ld) * kLower);
      }
    } else if (OUT && first > 0) {
      from(stored(p, kBegins, run, h), kLower);
    } else if (OUT && on) {
      from(stored(p, kFirst, run, h), kLower);
    } else if (kept && s.place0 > 0 && first == 0) {
#pragma unroll
      for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          S[a][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(state, in_state, row_of(a, r), 0)) *
                    (OUT ? kLower : 1.f);
    }
    // (the run that stores the sequence's last state may do so before another looks at what the slot holds)
    if (!OUT && first == 0) into(stored(p, kFirst, run, h));
    // What a run adds to its last sequence is a sum in any order: from the last chunk to the first, so that outputs,
    // which begin with the first ones, find those keys and values in the last-level cache (eight long prompts 559 ->
    // 538 us; of 760 MB it holds a third).
    int t0 = OUT ? first : last - kChunk;  // (a run's last sequence that goes on has whole chunks)
    fetch(t0);
    int age = 0;
    if (!OUT && first == 0) {
      const float fade = power(float(last) * ld);
#pragma unroll
      for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) S[a][r] *= fade;
    }
    for (int i = 0; i < chunks; ++i, t0 += OUT ? kChunk : -kChunk) {
      const int len = min(kChunk, last - t0);
      // Outputs: S, whatever the text says of it, is kept as of `age` tokens ago (without their decay), so that it is
      // not multiplied with every chunk's; what is added to it is raised by as much.  And times kLower.
      const bool renew = OUT && float(age + len) * ld < -kRaised;
      const int from_age = renew ? -len : age;
      if (threadIdx.x < kChunk)
        weight[threadIdx.x] = power(float(OUT ? -(from_age + 1 + min(int(threadIdx.x), len - 1))
                                              : last - 1 - t0 - int(threadIdx.x)) * ld) * (OUT ? kLower : 1.f);
      store_columns(kt, nk);
      store_columns(vt, nv);
      if constexpr (OUT) {
        store_rows(ks, nk);
        store_rows(qs, nq);
      }
      lds_barrier();
      if (i + 1 < chunks) fetch(t0 + (OUT ? kChunk : -kChunk));
      // (what is worked out from these is not worth a register from chunk to chunk)
      int row = c, four = 4 * g;
      asm volatile("" : "+v"(my_row), "+v"(my_col), "+v"(my_sc), "+v"(ld), "+v"(row), "+v"(four));
      uint16_t* const out = OUT ? static_cast<uint16_t*>(p.out) + (s.start + t0) * p.out_stride + h * D + b0 : nullptr;
      u32x4 vf[4];
      auto read_values = [&] {
#pragma unroll
        for (int k = 0; k < 4; ++k) vf[k] = read_col(vt, wave, k);
      };
      if constexpr (OUT) {
        // Scores of 32 x 32 (tokens down, queries across), three of the chunk's four:
        // (0, 0), (32, 32), and (0, 32).
        f32x16 X[kMine];
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
          const int tile = wave + m * W;
          if (tile < 3) {
            X[m] = f32x16{};
            const int kr = my_row + (tile == 1 ? 32 * kRow : 0), qr = my_row + (tile != 0 ? 32 * kRow : 0);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) X[m] = mfma(read(kr ^ 32 * k, ks), read(qr ^ 32 * k, qs), X[m]);
          }
        }
        lds_barrier();
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
          const int tile = wave + m * W;
          if (tile < 3) {
            const int kr = tile == 1, qr = tile != 0;
            const int gap = 32 * (qr - kr) + row - four;  // to the token of element 8 q + e: 8 q + e less
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float v[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = gap >= 8 * q + e ? X[m][4 * q + e] * by_gap[m][4 * q + e] : 0.f;
              const int to = (my_sc ^ 4 * four ^ 16 * (4 * kr + q)) + 2 * four + 32 * qr * kCol;
              const uint32_t lo = cut(v[0], v[1]), hi = cut(v[2], v[3]);
              write8(to, sc, lo, hi);
              write8(to, sc + 64 * kCol, pair(v[0], v[1]), pair(v[2], v[3]));
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
              const uint32_t v = __float_as_uint(S[a][8 * kk + 2 * e]), w = __float_as_uint(S[a][8 * kk + 2 * e + 1]);
              hi[e] = __builtin_amdgcn_perm(w, v, 0x07060302);
              lo[e] = pair(__uint_as_float(v) - __uint_as_float(v & 0xffff0000u),
                           __uint_as_float(w) - __uint_as_float(w & 0xffff0000u));
            }
            const u32x4 q0 = read_row(qs, 0, 2 * a + kk), q1 = read_row(qs, 1, 2 * a + kk);
            O[0] = mfma(hi, q0, O[0]);
            O[1] = mfma(hi, q1, O[1]);
            O[0] = mfma(lo, q0, O[0]);
            O[1] = mfma(lo, q1, O[1]);
          }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float f = power(float(age + 32 * i + row + 1) * ld) * kHigher;
#pragma unroll
          for (int r = 0; r < 16; ++r) O[i][r] = O[i][r] * f * p.scale;
        }
        lds_barrier();
        read_values();
        // A value that is no number (its product with zero is not zero) must not reach the
        // rows before its token through their scores of zero: it is left out of the
        // product, and put into the rows from its token on.
        float none = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) none = dot2(vf[k][e], zero, none);
        const bool odd = __ballot(none != 0.f) != 0;
        if (odd) {
          int token = kChunk;
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 7; e >= 0; --e) {
              const uint32_t half = e % 2 ? 0x7f800000u : 0x7f80u;
              if ((vf[k][e / 2] & half) == half) {
                token = min(token, 16 * k + 2 * four + e);
                vf[k][e / 2] &= e % 2 ? 0xffffu : 0xffff0000u;
              }
            }
          strange[b0 + c] = kChunk;
          __builtin_amdgcn_wave_barrier();
          atomicMin(&strange[b0 + c], token);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            if (k < 2) O[0] = mfma(vf[k], read_sc(part, 0, k), O[0]);
            O[1] = mfma(vf[k], read_sc(part, 1, k), O[1]);
          }
        }
        if (odd) {
          __builtin_amdgcn_wave_barrier();
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int token = strange[b0 + 8 * (r / 4) + four + r % 4];
#pragma unroll
            for (int i = 0; i < 2; ++i) O[i][r] = 32 * i + row >= token ? __uint_as_float(0x7fc00000u) : O[i][r];
          }
          read_values();
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (32 * i + row < len) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
              *reinterpret_cast<u32x2*>(out + (32 * i + row) * p.out_stride + 8 * q + four) =
                  u32x2{pair(O[i][4 * q], O[i][4 * q + 1]), pair(O[i][4 * q + 2], O[i][4 * q + 3])};
          }
      } else {
        read_values();
      }
      if (renew) {
        const float fade = power(float(age + len) * ld);
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
          for (int r = 0; r < 16; ++r) S[a][r] *= fade;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        u32x4 part[3];
        f32x4 w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) w[e] = *reinterpret_cast<const f32x4*>(weight + 16 * k + 2 * four + 4 * e);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float lo = bf16_lo(vf[k][e]) * w[e / 2][e % 2 * 2], hi = bf16_hi(vf[k][e]) * w[e / 2][e % 2 * 2 + 1];
          part[0][e] = cut(lo, hi), part[1][e] = cut(lo, hi);
          part[2][e] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);
        }
        u32x4 kf[NA];
#pragma unroll
        for (int a = 0; a < NA; ++a) kf[a] = read_col(kt, a, k);
#pragma unroll
        for (int i = 0; i < 3; ++i)
#pragma unroll
          for (int a = 0; a < NA; ++a) S[a] = mfma(kf[a], part[i], S[a]);
      }
      lds_barrier();
      age = from_age + len;
    }
    if constexpr (OUT) {
      const float fade = power(float(age) * ld) * kHigher;
#pragma unroll
      for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) S[a][r] *= fade;
    }

    if constexpr (!OUT) {
      into(stored(p, kBegins, run + 1, h));
      goes_on = first == 0 ? -chunks : chunks;
    } else if (kept && !on) {
#pragma unroll
      for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[a][r]), state, in_state, row_of(a, r), 0);
    }
    if (!OUT) break;
    ++b, at = 0;
  }
  if (!OUT && h == 0 && threadIdx.x == 0) p.goes_on[run] = goes_on;
}

// The states that runs begin with, from what the runs before them add: four
// numbers a thread.
template <int D>
__global__ __launch_bounds__(256) void k_decay_join(DecayArgs p) {
  constexpr int kParts = D * D / 4 / 256;  // workgroups of a head
  const int part = blockIdx.x % kParts, h = blockIdx.x / kParts;
  const float fade = log2_decay(p, h) * kChunk;
  f32x4* to = reinterpret_cast<f32x4*>(stored(p, kBegins, 1, h)) + part * 256 + threadIdx.x;
  const int64_t next = int64_t(p.states.heads) * (D * D / 4);
  f32x4 S = {};
  constexpr int kAtOnce = 8;  // runs whose sums are asked for together
  for (int run = 0; run + 1 < p.runs; run += kAtOnce, to += kAtOnce * next) {
    f32x4 x[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
      if (run + i + 1 < p.runs) x[i] = to[i * next];  // (whatever is there, if there is none)
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int chunks = run + i + 1 < p.runs ? p.goes_on[run + i] : 0;
      if (chunks > 0) {  // (a sequence that begins in the run has what it began with in the sum)
        const float f = exp2f(float(chunks) * fade);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][e] = fmaf(S[e], f, x[i][e]);
        to[i * next] = x[i];
      }
      S = x[i];
    }
  }
}

template <int D>
hipError_t prompt(const DecayArgs& p, hipStream_t s) {
  auto grid = [&](int runs) {  // (whole turns of the XCDs, each of heads that share a key head)
    return dim3((uint32_t(runs) * (p.states.heads / p.group) + kXcds - 1) / kXcds * kXcds * p.group);
  };
  if (p.runs > 1) {
    hipLaunchKernelGGL((k_decay_prompt<D, false>), grid(p.runs), dim3(2 * D), 0, s, p);
    if (p.join) hipLaunchKernelGGL((k_decay_join<D>), dim3(p.states.heads * (D * D / 1024)), dim3(256), 0, s, p);
  }
  hipLaunchKernelGGL((k_decay_prompt<D, true>), grid(p.runs ? p.runs : p.batch.batch), dim3(2 * D), 0, s, p);
  return hipGetLastError();
}

}  // namespace

// Token after token up to 8 of a sequence.  With states that come from memory, 28 heads, token
// after token and in a chunk (us): 5, 8 and 16 tokens of one sequence 7.7 and 10.1, 10.3 and 10.2,
// 17.2 and 10.2; of 64 sequences 55 and 60, 63 and 61, 87 and 64; with heads of 64 elements
// 5.0 and 7.1, 6.4 and 7.0, 10.0 and 7.1; 21 and 29, 24 and 29, 34 and 30.
//
// Then a workgroup to a sequence and head, or to a run of chunks of all sequences.
// What a chunk takes was measured (us), where a CU has one workgroup, two or three:
// 5.4 and 8.4 with heads of 128 elements (more do not fit), 3.3, 4.5 and 5.3 with 64.
// Runs cost another launch, the states that go from run to run (64 or 16 KiB a run
// and head, three times), and the keys' and values' chunks of every sequence that goes
// on in another run a second time (0.4 of a chunk).  The states that runs begin with are
// sums over the runs before: each run adds up its own (64 KiB of every run before it,
// 0.5 us where a CU has one workgroup, 0.9 with two), or, where those are many, a
// launch between the two does.  Measured on the side that the rule takes and on the other
// (28 heads of 128 elements, rows and states from memory): whole or in runs, 200 tokens 23.5
// and 23.6 us, 8 x 200 31 and 48, 3 x 300 32 and 36, 16 x 600 94 and 131, 8 x 6562 509 and
// 548; in runs or whole, 330 tokens 25.6 and 33, 1286 tokens 37.5 and 105, four of 2000 109 and
// 160, 9459 135 and 696, eight of 3531 to 9459 553 and 686; sums of their own or joined,
// 1286 tokens 37.4 and 40.5, eight of 3531 to 9459 553 and 559; joined or not, 9459 tokens
// 135 and 142.  With heads of 64 elements, whole or in runs: 64 x 600 161 and 175, 32 x 3000
// 408 and 427; in runs or whole: 1286 tokens 25.6 and 72, 8 x 3000 124 and 157; joined or
// not, 9459 tokens 69.1 and 67.2.
DecayPlan decay_plan(const wz_states& z, const wz_ragged& r) {
  DecayPlan p{};
  p.token = r.max_tokens <= 8;
  if (p.token) return p;
  const double most = (r.max_tokens + kChunk - 1) / kChunk;
  // chunks of all sequences at most
  const double all = std::min(r.batch * most, double(r.tokens / kChunk + r.batch));
  struct Times {
    double alone, full;     // a chunk: of a CU's only workgroup; a CU's time for one, with as many as fit
    int at_once;            // workgroups of a CU
    double chunk[4];        // a chunk with 1, 2, ... of them
    double adds[4];         // what one run before adds, with 1, 2, ...
    double join, join_run;  // a launch that adds up; for each run
  };
  static constexpr Times k128{4.9, 3.9, 2, {0, 5.4, 8.4}, {0, 0.5, 0.9}, 6, 0.2};
  static constexpr Times k64{3.15, 2.2, 3, {0, 3.3, 4.5, 5.3}, {0, 0.25, 0.35, 0.4}, 6, 0.1};
  const Times& x = z.head_dim == 128 ? k128 : k64;
  double best = 5 + std::max(most * x.alone, all * z.heads / kCUs * x.full);
  for (int n = x.at_once; n >= 0; --n) {  // (0: on half of the CUs)
    const int most_runs = std::min((n ? n * kCUs : kCUs / 2) / z.heads, int(all / 2));
    if (most_runs < 2) continue;
    const double each = std::ceil(all / most_runs), again = std::max(0., 1 - each * r.batch / (2 * all));
    const int runs = int(std::ceil(all / each)), there = (runs * z.heads + kCUs - 1) / kCUs;
    const double join = x.join + x.join_run * runs, adds = x.adds[there] * std::min(std::ceil(most / each), runs - 1.);
    const double next = 12 * each * r.batch / all;  // from one sequence to the next
    const double states = 0.025 * runs * z.heads * z.head_dim * z.head_dim / 16384;  // to memory and from it
    const double time = 5 + states + std::min(join, adds) + each * x.chunk[there] * (1 + 0.4 * again) + next;
    if (time < best) best = time, p.runs = runs, p.join = join < adds;
  }
  if (p.runs == 0) return p;
  p.state_bytes = size_t(2) * p.runs * z.heads * z.head_dim * z.head_dim * 4;
  p.bytes = p.state_bytes + (size_t(p.runs) * 4 + 255) / 256 * 256;
  return p;
}

hipError_t launch_decay_prompt(const DecayArgs& p, hipStream_t s) {
  return p.states.head_dim == 128 ? prompt<128>(p, s) : prompt<64>(p, s);
}

}  // namespace wz
