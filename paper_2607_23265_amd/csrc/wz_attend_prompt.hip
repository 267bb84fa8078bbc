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
#include "wz_attend.h"

namespace wz {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kRows = 32 * kWaves;

// A running maximum is followed only once it is passed by this much (in powers
// of two): the sums are rescaled on few tiles, and probabilities stay below 2^8.
constexpr float kSlack = 8.f;

// Classes of instructions for the scheduler.
constexpr int kVector = 0x2, kProducts = 0x8;

template <int D>
struct Stages {
  __bf16 k[2][kTile * D];  // [row of a product][D]
  __bf16 v[2][D * kTile];  // [channel][token]
};

// Tiles [off, off + count) of block kb of sequence b, key/value head h; slot:
// where its part goes, -1 if the block is this workgroup's alone.
template <int D>
__device__ __forceinline__ void attend_block(const AttendArgs& a, const Partition<kRows>& part, int h, int b, int kb,
                                             int off, int count, int slot, Stages<D>& lds) {
  constexpr int KK = D / 16, DT = D / 32, kExchange = D / 8 - 1;
  constexpr int kKeyPieces = kTile * (D / 16) / kThreads, kValPieces = D * (kTile / 16) / kThreads;
  auto& kt = lds.k;
  auto& vt = lds.v;
  const int Hkv = a.cache.kv_heads, G = part.G;
  const Seq s = sequence(a.batch, b);
  const Block blk = part.block(s, kb);
  const int T0 = blk.lo / kTile + off;
  const int T1 = min((max(blk.hi, blk.lo) + kTile - 1) / kTile, T0 + count);

  const int tid = threadIdx.x, lane = __lane_id(), w = tid / kWave, c = lane & 31, g = lane >> 5;
  const int P = a.cache.page_size, logP = __builtin_ctz(P);
  const uint8_t* const kc = static_cast<const uint8_t*>(a.cache.k);
  const uint8_t* const vc = static_cast<const uint8_t*>(a.cache.v);

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

  // Staging: this thread's pieces of a tile, 16 codes each.  Nothing branches
  // around a load: what lies behind the last tile is the last tile again, and a
  // block of 16 tokens that has no page reads page 0 and is masked.
  u32x4 kx[kKeyPieces], vx[kValPieces];
  float ks[kKeyPieces], vs;
  uint32_t in_next = 0;  // bit k: tokens 16 k .. of the tile loaded last lie in pages of the cache
  struct Pages {
    int k[kKeyPieces], v;
  } ids;
  const int* const row_of = a.batch.table + int64_t(b) * a.batch.table_stride;
  const int entries = max((s.kv + P - 1) >> logP, 1);
  auto pages = [&](int tile) {
    const int tok = min(tile, T1 - 1) * kTile;
    Pages x;
#pragma unroll
    for (int i = 0; i < kKeyPieces; ++i)
      x.k[i] = row_of[min((tok + (tid + i * kThreads) / (D / 16) / 16 * 16) >> logP, entries - 1)];
    x.v = row_of[min((tok + 16 * (tid % 4)) >> logP, entries - 1)];
    return x;
  };
  auto load = [&](int tile, const Pages& id) {
    const int first = min(tile, T1 - 1) * kTile;
    const bool vin = uint32_t(id.v) < uint32_t(a.cache.pages);
    in_next = uint32_t(__ballot(vin)) & 0xfu;
#pragma unroll
    for (int i = 0; i < kKeyPieces; ++i) {
      const int p = tid + i * kThreads, tok = p / (D / 16), part16 = p % (D / 16);
      const int64_t at = int64_t(uint32_t(id.k[i]) < uint32_t(a.cache.pages) ? id.k[i] : 0) * Hkv + h;
      kx[i] = *reinterpret_cast<const u32x4*>(kc + at * (P * D) + ((first + tok) & (P - 1)) * D + 16 * part16);
      ks[i] = a.cache.k_scale[at];
    }
    const int64_t at = int64_t(vin ? id.v : 0) * Hkv + h;
    const float scale = a.cache.v_scale[at];
    vs = vin ? scale : 1.f;
#pragma unroll
    for (int i = 0; i < kValPieces; ++i) {
      const int p = tid + i * kThreads, d = p / 4;
      vx[i] = *reinterpret_cast<const u32x4*>(vc + at * (P * D) + d * P + ((first + 16 * (p % 4)) & (P - 1)));
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // values behind the sequence's end may be any bytes and must be zeros
  auto cut = [&](int tile) {
    const int first = min(tile, T1 - 1) * kTile;
    if (first + kTile > s.kv || in_next != 0xfu) {
      const int count = in_next >> (tid % 4) & 1u ? min(max(s.kv - (first + 16 * (tid % 4)), 0), 16) : 0;
#pragma unroll
      for (int i = 0; i < kValPieces; ++i) vx[i] = first_codes(vx[i], count);
    }
  };
  auto store_piece = [&](int buf, int i) {  // keys' pieces, then values'
    if (i < kKeyPieces) {
      const int p = tid + i * kThreads, tok = p / (D / 16), part16 = p % (D / 16);
      const int r = (tok & 32) | (tok & 16) | (tok & 4) << 1 | (tok & 8) >> 1 | (tok & 3);
      __bf16* at = kt[buf] + r * D;
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * part16) ^ (r & kExchange))) = decode8(kx[i][0], kx[i][1], ks[i]);
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * part16 + 1) ^ (r & kExchange))) = decode8(kx[i][2], kx[i][3], ks[i]);
    } else if (i < kKeyPieces + kValPieces) {
      const int k = i - kKeyPieces, p = tid + k * kThreads, d = p / 4, part16 = p % 4;
      __bf16* at = vt[buf] + d * kTile;
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * part16) ^ (d >> 1 & 7))) = decode8(vx[k][0], vx[k][1], vs);
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * part16 + 1) ^ (d >> 1 & 7))) = decode8(vx[k][2], vx[k][3], vs);
    }
  };
  static_assert(kKeyPieces + kValPieces <= KK / 2, "a piece is stored with every batch of products");

  uint32_t in = 0, in_stored = 0;
  if (T0 < T1) {
    const Pages now = pages(T0), then = pages(T0 + 1);
    ids = pages(T0 + 2);
    load(T0, now);
    cut(T0);
#pragma unroll
    for (int i = 0; i < kKeyPieces + kValPieces; ++i) store_piece(0, i);
    in = in_next;
    load(T0 + 1, then);
  }
  for (int tile = T0; tile < T1; ++tile) {
    const int buf = (tile - T0) & 1;
    __syncthreads();
    cut(tile + 1);
    // Scores.  Fragments are read from LDS four at a time, one batch ahead of
    // its products; the next tile, which has arrived, goes to the other buffer
    // between them.
    f32x16 sc[2] = {};
    bf16x8 f[2][4];
    const __bf16* const keys = kt[buf] + c * D;
    auto read_keys = [&](int j) {  // batch j of KK / 2: products 4 j .. 4 j + 3, by 32 tokens and then by 16 channels
#pragma unroll
      for (int i = 0; i < 4; ++i)
        f[j % 2][i] = *reinterpret_cast<const bf16x8*>(keys + (4 * j + i) / KK * 32 * D +
                                                       8 * ((2 * ((4 * j + i) % KK) + g) ^ (c & kExchange)));
      __builtin_amdgcn_sched_barrier(0);
    };
    read_keys(0);
#pragma unroll
    for (int j = 0; j < KK / 2; ++j) {
      if (j + 1 < KK / 2) read_keys(j + 1);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sc[(4 * j + i) / KK] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[j % 2][i], qf[(4 * j + i) % KK],
                                                                       sc[(4 * j + i) / KK], 0, 0, 0);
      store_piece(buf ^ 1, j);
      __builtin_amdgcn_sched_barrier(0);
    }
    in_stored = in_next;
    {
      const Pages now = ids;
      ids = pages(tile + 3);
      load(tile + 2, now);
    }
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
    if (__any(top > m + kSlack)) {
      const float mx = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - (mx == -INFINITY ? 0.f : mx));
      l *= f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= f;
      m = mx;
    }
    const float use = m == -INFINITY ? 0.f : m;
    // Products with the values, 16 tokens at a time, the probabilities of the
    // next 16 between them.
    bf16x8 p[2], v[2][DT];
    auto read_values = [&](int u) {
#pragma unroll
      for (int d = 0; d < DT; ++d)
        v[u % 2][d] = *reinterpret_cast<const bf16x8*>(vt[buf] + (32 * d + c) * kTile + 8 * ((2 * u + g) ^ (c >> 1 & 7)));
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
  }
  {
    const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(u[0]) + __uint_as_float(u[1]);
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

template <int D>
__global__ __launch_bounds__(kThreads, 2) void k_attend_prompt(AttendArgs a) {
  __shared__ __align__(16) Stages<D> lds;
  const int Hkv = a.cache.kv_heads, h = blockIdx.x % Hkv, all = gridDim.x / Hkv;
  const Partition<kRows> part(a);
  // the last blocks first: in a causal batch they are the longest
  part.each_piece(all - 1 - int(blockIdx.x) / Hkv, [&](int b, int k, int off, int count, int slot) {
    attend_block<D>(a, part, h, b, k, off, count, slot, lds);
  });
}

}  // namespace

hipError_t launch_attend_prompt(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  const dim3 grid(uint32_t((p.shared ? p.workers : p.blocks) * a.cache.kv_heads)), block(kThreads);
  if (a.cache.head_dim == 128) hipLaunchKernelGGL((k_attend_prompt<128>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_attend_prompt<64>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace wz
