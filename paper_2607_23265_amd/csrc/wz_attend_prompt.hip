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
// 16-byte chunks of a row in LDS are exchanged by the row's last three bits, so
// that eight lanes that read eight rows hit all banks.
#include "wz_attend.h"

namespace wz {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kRows = 32 * kWaves;

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
  constexpr int KK = D / 16, DT = D / 32;
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
  bf16x8 qf[KK];
  {
    const uint16_t* src =
        static_cast<const uint16_t*>(a.q) + int64_t(s.start + row / G) * a.q_stride + (h * G + row % G) * D + 8 * g;
#pragma unroll
    for (int k = 0; k < KK; ++k) qf[k] = valid ? *reinterpret_cast<const bf16x8*>(src + 16 * k) : bf16x8{};
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
    const int first = tile * kTile;
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
  auto store = [&](int buf, int tile) {
    // values behind the sequence's end may be any bytes and must be zeros
    if (tile * kTile + kTile > s.kv || in_next != 0xfu) {
      const int count = in_next >> (tid % 4) & 1u ? min(max(s.kv - (tile * kTile + 16 * (tid % 4)), 0), 16) : 0;
#pragma unroll
      for (int i = 0; i < kValPieces; ++i) vx[i] = first_codes(vx[i], count);
    }
#pragma unroll
    for (int i = 0; i < kKeyPieces; ++i) {
      const int p = tid + i * kThreads, tok = p / (D / 16), part16 = p % (D / 16);
      const int r = (tok & 32) | (tok & 16) | (tok & 4) << 1 | (tok & 8) >> 1 | (tok & 3);
      __bf16* at = kt[buf] + r * D;
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * part16) ^ (r & 7))) = decode8(kx[i][0], kx[i][1], ks[i]);
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * part16 + 1) ^ (r & 7))) = decode8(kx[i][2], kx[i][3], ks[i]);
    }
#pragma unroll
    for (int i = 0; i < kValPieces; ++i) {
      const int p = tid + i * kThreads, d = p / 4, part16 = p % 4;
      __bf16* at = vt[buf] + d * kTile;
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * part16) ^ (d & 7))) = decode8(vx[i][0], vx[i][1], vs);
      *reinterpret_cast<bf16x8*>(at + 8 * ((2 * part16 + 1) ^ (d & 7))) = decode8(vx[i][2], vx[i][3], vs);
    }
  };

  uint32_t in = 0;
  if (T0 < T1) {
    const Pages now = pages(T0);
    ids = pages(T0 + 1);
    load(T0, now);
    in = in_next;
    store(0, T0);
  }
  for (int tile = T0; tile < T1; ++tile) {
    const int buf = (tile - T0) & 1;
    __syncthreads();
    const bool more = tile + 1 < T1;
    if (more) {
      const Pages now = ids;
      ids = pages(tile + 2);
      load(tile + 1, now);
    }
    f32x16 sc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      sc[t] = f32x16{};
      const __bf16* at = kt[buf] + (32 * t + c) * D;
#pragma unroll
      for (int k = 0; k < KK; ++k)
        sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            *reinterpret_cast<const bf16x8*>(at + 8 * ((2 * k + g) ^ (c & 7))), qf[k], sc[t], 0, 0, 0);
    }
    const bool masked = tile * kTile < blk.full_lo || tile * kTile + kTile > blk.full_hi || in != 0xfu;
#pragma unroll
    for (int t = 0; t < 2; ++t) sc[t] *= a.scale2;
    if (masked) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = tile * kTile + 32 * t + 16 * (i / 8) + 8 * g + i % 8;
          sc[t][i] = j >= lo && j < hi && (in >> (2 * t + i / 8) & 1u) ? sc[t][i] : -INFINITY;
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[t][i]);
    {
      const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1]));
    }
    const float mx = fmaxf(m, top), use = mx == -INFINITY ? 0.f : mx;
    if (__any(mx > m)) {
      const float f = __builtin_amdgcn_exp2f(m - use);
      l *= f;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= f;
    }
    m = mx;
#pragma unroll
    for (int u = 0; u < 4; ++u) {  // 16 tokens
      bf16x8 p;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = __builtin_amdgcn_exp2f(sc[u / 2][8 * (u % 2) + i] - use);
        l += e;
        p[i] = __bf16(e);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d)
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            *reinterpret_cast<const bf16x8*>(vt[buf] + (32 * d + c) * kTile + 8 * ((2 * u + g) ^ (c & 7))), p, o[d], 0,
            0, 0);
    }
    if (more) store(buf ^ 1, tile + 1);
    in = in_next;
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
