// Attention of many rows over the 8-bit cache (wz_cache_attention with more
// than 64 rows to a key/value head of a sequence: prompts).
//
// Four waves share a block of 128 rows, 32 each, and every tile of 64 tokens,
// which lies in LDS as bf16: the codes of the next tile are loaded while this
// one is worked on, decoded (times their page's scale: exact) and put into the
// other of two buffers.  The products are the transposed ones of the token
// kernel, 32 x 32 x 16:
//
//   S^T = K Q^T   row r of a product is token 16 (r / 16) + 8 (r / 4 % 2) + 4 (r /
//                 8 % 2) + r % 4 of its 32 (keys lie in LDS in that order), so
//                 that a lane of column c and half g ends with the scores of tokens
//                 16 u + 8 g .. + 7 together: its right operands of
//   O^T = V^T P   as they stand.  A column's maximum and sum are a lane's own
//                 and one swap of halves.
//
// 16-byte chunks of a row in LDS are exchanged by the row's number, so that
// sixteen lanes that read sixteen rows hit all 64 banks.
//
// Measured: 1.19 TFLOP of two causal prompts of 8 300 to 9 459 tokens, 28 heads of
// 128 over 4, in 1129 to 1161 us on different cards (1.05 to 1.03 PFLOP/s; the
// library's 8192^3 bf16 product 1.53).
// A wave of 32 rows fills the registers of two waves a SIMD (output 64, scores
// 32, queries 32, fragments 64), and those two must overlap vector work, 60 % of
// the cycles, with products, 50 %; LDS is at 38 %, without conflicts.  128 rows
// share a decoded tile because two workgroups then fit a CU and wait apart:
// eight waves in one took 1330 us where four took 1246.
#include "wz_attend.h"

namespace wz {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4;  // of a group
constexpr int kThreads = kWaves * kWave;
constexpr int kRows = 32 * kWaves;

// Classes of instructions for the scheduler.
constexpr int kVector = 0x2, kScalar = 0x4, kProducts = 0x8;

template <int D>
struct Stages {
  __bf16 k[2][kTile * D];  // [row of a product][D]
  __bf16 v[2][D * kTile];  // [channel][token]
};

// A value row (128 bytes of 256 of banks) exchanges its chunks so that eight
// lanes that write eight rows and sixteen that read sixteen meet no bank twice.
__device__ __forceinline__ int value_exchange(int channel) { return (channel & 7) ^ (channel >> 3 & 1); }

// `count` tiles from spot x on, key/value head h; slot: where their part goes, -1
// if the block is this workgroup's alone.
// KG groups of four waves take the tiles in turn, each with stages of its own,
// and add up at the end.
template <int D, int KG>
__device__ __forceinline__ void attend_block(const AttendArgs& a, const Partition<kRows>& part, int h, const Spot& x,
                                             int count, int slot, Stages<D> (&stages)[KG]) {
  constexpr int KK = D / 16, DT = D / 32, kExchange = D / 8 - 1;
  constexpr int kKeyPieces = kTile * (D / 16) / kThreads, kValPieces = D * (kTile / 16) / kThreads;
  const int Hkv = a.cache.kv_heads, G = part.G;
  const Seq s = x.s;
  const Block blk = part.block(s, x.k);
  const int T0 = blk.lo / kTile + x.off;
  const int T1 = min((max(blk.hi, blk.lo) + kTile - 1) / kTile, T0 + count);

  const int lane = __lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int w = wave % kWaves, group = wave / kWaves, tid = threadIdx.x % kThreads;
  auto& kt = stages[group].k;
  auto& vt = stages[group].v;
  const int c = lane & 31, g = lane >> 5;
  const int P = a.cache.page_size, logP = __builtin_ctz(P);

  const int row = blk.r0 + 32 * w + c;
  const bool valid = row < blk.rows;
  int lo, hi;
  row_range(a, s, row, G, &lo, &hi);
  if (!valid) hi = 0;
  // scores are compared before they are scaled, so the factor's sign goes to
  // the query (exact)
  const float scale2 = fabsf(a.scale2);
  const uint32_t flip = a.scale2 < 0.f ? 0x80008000u : 0u;
  bf16x8 qf[KK];
  {
    const uint16_t* src =
        static_cast<const uint16_t*>(a.q) + int64_t(s.start + row / G) * a.q_stride + (h * G + row % G) * D + 8 * g;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      u32x4 u{};
      if (valid) u = *reinterpret_cast<const u32x4*>(src + 16 * k);
      qf[k] = __builtin_bit_cast(bf16x8, u ^ flip);
    }
  }
  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = f32x16{};
  float m = -INFINITY, l = 0.f;

  // Staging: this wave's pieces of a tile, 16 codes a lane.  A piece is of one
  // block of 16 tokens, so its page and scale are the same in the whole wave and
  // its lanes' offsets never change.  Nothing branches around a load: what lies
  // behind the last tile is the last tile again, and a block that has no page
  // reads page 0 and is masked.
  u32x4 kx[kKeyPieces], vx[kValPieces];
  float ks4 = 0.f, vs4 = 0.f;  // scales of block lane % 4
  uint32_t in_next = 0;        // bit k: block k of the tile loaded last lies in a page of the cache
  const int* const row_of = a.batch.table + int64_t(x.seq) * a.batch.table_stride;
  const int entries = max((s.kv + P - 1) >> logP, 1);
  // LDS takes eight lanes' 16 bytes at once, over 128 bytes of banks.  A lane's
  // two chunks are next to each other, so eight lanes hold four pieces each of
  // two rows, which the exchange sends to even and to odd chunks.
  const int ktok = tid / (D / 8) * 2 + (tid >> 2 & 1), kpart = (tid & 3) | (tid % (D / 8) >> 3 << 2);
  const uint32_t koff = (ktok & 15) * D + 16 * kpart, voff = lane * P;
  auto key_block = [&](int i) { return (w * kWave + i * kThreads) / D; };  // (tok / 16)
  const uint32_t page_bytes = uint32_t(Hkv) * P * D;  // of all heads
  const uint8_t* const kbase = static_cast<const uint8_t*>(a.cache.k) + uint32_t(h) * P * D;
  const uint8_t* const vbase = static_cast<const uint8_t*>(a.cache.v) + uint32_t(h) * P * D;
  auto pages = [&](int tile) {  // of block lane % 4
    return row_of[min((min(tile, T1 - 1) * kTile + 16 * (lane & 3)) >> logP, entries - 1)];
  };
  // The page of block lane % 4 of a tile, and its scales, asked for: worked out
  // in lanes, between products, since a wave waits for every step of a chain of
  // scalar instructions (prompts of two long videos 1223 -> 1193 us).
  struct Next {
    uint64_t page;  // its first byte
    float ks, vs;
    uint32_t in;
  };
  auto find = [&](int id) {
    Next n;
    const bool there = uint32_t(id) < uint32_t(a.cache.pages);
    n.in = uint32_t(__ballot(there)) & 0xfu;
    const uint32_t page = there ? id : 0;
    n.page = uint64_t(page) * page_bytes;
    const uint64_t scale_at = uint64_t(page) * uint32_t(Hkv);
    n.ks = a.cache.k_scale[scale_at + h], n.vs = a.cache.v_scale[scale_at + h];
    return n;
  };
  auto lane_of64 = [](uint64_t x, int i) {
    const uint32_t lo = __builtin_amdgcn_readlane(uint32_t(x), i), hi = __builtin_amdgcn_readlane(uint32_t(x >> 32), i);
    return uint64_t(hi) << 32 | lo;
  };
  auto load_piece = [&](int tile, const Next& n, int i) {  // keys' pieces, then values'
    const uint32_t first = min(tile, T1 - 1) * kTile;
    if (i < kKeyPieces) {
      const uint32_t in_page = ((first + 16 * key_block(i)) & (P - 1)) * D;
      kx[i] = *reinterpret_cast<const u32x4*>(kbase + lane_of64(n.page, key_block(i)) + (in_page + koff));
    } else if (i < kKeyPieces + kValPieces) {
      const int k = i - kKeyPieces;
      const uint32_t in_page = (first + 16 * w) & (P - 1);
      vx[k] = *reinterpret_cast<const u32x4*>(vbase + lane_of64(n.page, w) + (in_page + 64 * k * P + voff));
    }
  };
  auto loaded = [&](const Next& n) { ks4 = n.ks, vs4 = n.vs, in_next = n.in; };
  auto load = [&](int tile, const Next& n) {
#pragma unroll
    for (int i = 0; i < kKeyPieces + kValPieces; ++i) load_piece(tile, n, i);
    loaded(n);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto lane_of = [](float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); };
  // values behind the sequence's end may be any bytes and must be zeros
  auto cut = [&](int tile) {
    const int first = min(tile, T1 - 1) * kTile;
    if (first + kTile > s.kv || in_next != 0xfu) {
      const int count = in_next >> w & 1u ? min(max(s.kv - (first + 16 * w), 0), 16) : 0;
#pragma unroll
      for (int i = 0; i < kValPieces; ++i) vx[i] = first_codes(vx[i], count);
    }
  };
  auto store_piece = [&](int buf, int i) {  // keys' pieces, then values'
    if (i < kKeyPieces) {
      const int tok = ktok + i * (kThreads * 16 / D);
      const int r = (tok & 32) | (tok & 16) | (tok & 4) << 1 | (tok & 8) >> 1 | (tok & 3);
      const float scale = lane_of(ks4, key_block(i));
      __bf16* at = kt[buf] + r * D;
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * kpart) ^ (r & kExchange))) = decode8(kx[i][0], kx[i][1], scale);
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * kpart + 1) ^ (r & kExchange))) = decode8(kx[i][2], kx[i][3], scale);
    } else if (i < kKeyPieces + kValPieces) {
      const int k = i - kKeyPieces, d = lane + 64 * k;
      const float there = lane_of(vs4, w), scale = in_next >> w & 1u ? there : 1.f;
      __bf16* at = vt[buf] + d * kTile;
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * w) ^ value_exchange(d))) = decode8(vx[k][0], vx[k][1], scale);
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * w + 1) ^ value_exchange(d))) = decode8(vx[k][2], vx[k][3], scale);
    }
  };
  static_assert(kKeyPieces + kValPieces <= KK / 2, "a piece is stored with every batch of products");

  uint32_t in = 0;
  int ids = 0;
  Next next;
  // One tile, in buffer `buf` (known to the compiler, which turns it into
  // offsets of the instructions).
  auto turn = [&](int tile, auto buffer) {
    constexpr int buf = decltype(buffer)::value;
    __syncthreads();
    if (KG > 1 && tile >= T1) return;  // (the other group has one tile more)
    cut(tile + KG);
    // Scores.  Fragments are read from LDS four at a time, one batch ahead of
    // its products; the next tile, which has arrived, goes to the other buffer
    // between them.
    f32x16 sc[2] = {};
    bf16x8 f[2][4];
    const __bf16* const keys = kt[buf] + c * D;
    auto read_keys = [&](int j) {  // batch j of KK / 2: products 4 j .. 4 j + 3, the two halves of the tile in turn
#pragma unroll
      for (int i = 0; i < 4; ++i)
        f[j % 2][i] = *reinterpret_cast<const bf16x8*>(keys + i % 2 * 32 * D +
                                                       8 * ((2 * (2 * j + i / 2) + g) ^ (c & kExchange)));
      __builtin_amdgcn_sched_barrier(0);
    };
    read_keys(0);
#pragma unroll
    for (int j = 0; j < KK / 2; ++j) {
      if (j + 1 < KK / 2) read_keys(j + 1);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sc[i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[j % 2][i], qf[2 * j + i / 2], sc[i % 2], 0, 0, 0);
      // a piece's registers are free with its store, and a load that goes out
      // then has a whole turn to come back
      store_piece(buf ^ 1, j);
      load_piece(tile + 2 * KG, next, j);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kVector | kScalar, 5, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    const uint32_t in_stored = in_next;
    loaded(next);
    next = find(ids);
    ids = pages(tile + 4 * KG);
    __builtin_amdgcn_sched_barrier(0);
    if (tile * kTile < blk.full_lo || tile * kTile + kTile > blk.full_hi || in != 0xfu) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = tile * kTile + 32 * t + 16 * (i / 8) + 8 * g + i % 8;
          sc[t][i] = j >= lo && j < hi && (in >> (2 * t + i / 8) & 1u) ? sc[t][i] : -INFINITY;
        }
    }
    in = in_stored;
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[t][i]);
    {
      const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1])) * scale2;
    }
    // The maximum is followed at once: a row that one token dominates then has
    // that token's probability as exactly 1.  (Following it only when passed by
    // 2^8 saves 1.5 % of the time and costs a quarter more error against 64
    // bits, 0.0021 for 0.0017.)
    if (__any(top > m)) {
      const float mx = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - (mx == -INFINITY ? 0.f : mx));
      l *= f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= f;
      m = mx;
    }
    const float use = m == -INFINITY ? 0.f : m;
    // Products with the values, 16 tokens at a time, the probabilities of the
    // next 16 between them.  Each is rounded to bf16 once, for products at bf16's
    // rate with values that it holds exactly; the sum takes it unrounded (error
    // against 64 bits, of results in bf16: 0.0017 to 0.0018, with fp32
    // probabilities 0.0017).
    bf16x8 p[2], v[2][DT];
    auto read_values = [&](int u) {
#pragma unroll
      for (int d = 0; d < DT; ++d)
        v[u % 2][d] = *reinterpret_cast<const bf16x8*>(vt[buf] + (32 * d + c) * kTile +
                                                       8 * ((2 * u + g) ^ value_exchange(c)));
      __builtin_amdgcn_sched_barrier(0);
    };
    auto probabilities = [&](int u) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = __builtin_amdgcn_exp2f(fmaf(sc[u / 2][8 * (u % 2) + i], scale2, -use));
        l += e;
        p[u % 2][i] = __bf16(e);
      }
    };
    read_values(0);
    probabilities(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (u < 3) read_values(u + 1);
#pragma unroll
      for (int d = 0; d < DT; ++d)
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[u % 2][d], p[u % 2], o[d], 0, 0, 0);
      if (u < 3) probabilities(u + 1);
      // products and vector work in turn
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kVector, 32 / DT, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (T0 < T1) {
    const int first = T0 + group, now = pages(first), then = pages(first + KG);
    const int after = pages(first + 2 * KG);
    ids = pages(first + 3 * KG);
    load(first, find(now));
    cut(first);
#pragma unroll
    for (int i = 0; i < kKeyPieces + kValPieces; ++i) store_piece(0, i);
    in = in_next;
    load(first + KG, find(then));
    next = find(after);
    for (int tile = T0; tile < T1; tile += 2 * KG) {  // (the same number of turns in every group)
      turn(tile + group, std::integral_constant<int, 0>{});
      if (tile + KG < T1) turn(tile + KG + group, std::integral_constant<int, 1>{});
    }
  }
  {
    const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(u[0]) + __uint_as_float(u[1]);
  }
  if constexpr (KG > 1) {
    static_assert(KG == 2, "");
    __syncthreads();  // no stage is read any more: the second group leaves its sums in its own
    float* const mine = reinterpret_cast<float*>(&stages[1]) + w * (DT * 16 * kWave) + lane;
    __shared__ float ml[2][kThreads];
    if (group == 1) {
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) mine[(16 * d + i) * kWave] = o[d][i];
      ml[0][tid] = m, ml[1][tid] = l;
    }
    __syncthreads();
    if (group == 1) return;
    const float m1 = ml[0][tid], l1 = ml[1][tid], mx = fmaxf(m, m1);
    // (a group without a score has a sum of 0, or of NaN if every score was)
    const float f0 = m == -INFINITY ? l : __builtin_amdgcn_exp2f(m - mx);
    const float f1 = m1 == -INFINITY ? l1 : __builtin_amdgcn_exp2f(m1 - mx);
    l = (m == -INFINITY ? l : l * f0) + (m1 == -INFINITY ? l1 : l1 * f1);
    m = mx;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * f0 + mine[(16 * d + i) * kWave] * f1;
  }
  if (!valid) return;
  if (slot >= 0) {
    const int64_t at = (int64_t(slot) * Hkv + h) * kRows + 32 * w + c;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(a.part + at * D + 32 * d + 8 * i + 4 * g) =
            f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    if (g == 0) a.part_ml[2 * at] = m, a.part_ml[2 * at + 1] = l;
    return;
  }
  const int t = s.start + row / G, head = h * G + row % G;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint16_t* dst = static_cast<uint16_t*>(a.out) + t * a.out_stride + head * D;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x2*>(dst + 32 * d + 8 * i + 4 * g) =
          u32x2{to_bf16(o[d][4 * i] * inv) | uint32_t(to_bf16(o[d][4 * i + 1] * inv)) << 16,
                to_bf16(o[d][4 * i + 2] * inv) | uint32_t(to_bf16(o[d][4 * i + 3] * inv)) << 16};
  if (a.lse && g == 0) a.lse[int64_t(t) * a.q_heads + head] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
}

template <int D, int KG>
__global__ __launch_bounds__(KG* kThreads, 2) void k_attend_prompt(AttendArgs a) {
  __shared__ __align__(16) Stages<D> stages[KG];
  const int Hkv = a.cache.kv_heads, h = blockIdx.x % Hkv, all = gridDim.x / Hkv;
  const Partition<kRows> part(a);
  // the last blocks first: in a causal batch they are the longest
  part.each_piece(all - 1 - int(blockIdx.x) / Hkv, [&](const Spot& x, int count, int slot) {
    attend_block<D, KG>(a, part, h, x, count, slot, stages);
  });
}

template <int D>
void launch(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  const dim3 grid(uint32_t((p.shared ? p.workers : p.blocks) * a.cache.kv_heads));
  if (p.groups == 2) hipLaunchKernelGGL((k_attend_prompt<D, 2>), grid, dim3(2 * kThreads), 0, s, a);
  else hipLaunchKernelGGL((k_attend_prompt<D, 1>), grid, dim3(kThreads), 0, s, a);
}

}  // namespace

hipError_t launch_attend_prompt(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  if (a.cache.head_dim == 128) launch<128>(a, p, s);
  else launch<64>(a, p, s);
  return hipGetLastError();
}

}  // namespace wz
