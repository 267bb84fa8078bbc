// Attention of few rows over the 8-bit cache (wz_cache_attention with up to 64
// rows to a key/value head of a sequence: single tokens, tokens to verify),
// and the sum of shared blocks' parts.
//
// The work is one pass over the keys and values, so the kernel is made to keep
// loads in flight and nothing between them and the matrix instructions: no
// LDS, every load 16 bytes a lane in the order the fragments need.
//
//   S^T = K Q^T   16 x 16 x 32: rows are tokens, columns the query rows.  Row
//                 r of product t (t < 4) is token 16 (r / 4) + 4 t + r % 4 of the
//                 tile, so that a lane of column c and quarter q ends with the
//                 scores of tokens 16 q .. 16 q + 15 in order.
//   O^T = V^T P   the same lane's probabilities of tokens 16 q + 8 m + j are
//                 product m's right operand as they stand; its left operand is
//                 8 bytes of a channel's tokens, which lie together in a page.
//
// Four waves take a block's tiles in turn, each with a running maximum and sum,
// and join through LDS at the end in a fixed order.
#include "wz_attend.h"

namespace wz {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;

template <int D, int NT>
__global__ __launch_bounds__(kThreads) void k_attend_token(AttendArgs a, int blocks_bound) {
  constexpr int BR = 16 * NT, KK = D / 32, DT = D / 16, kPieces = D / 64;
  constexpr int kLd = D + 4;
  __shared__ float so[BR * kLd];
  __shared__ float sm[kWaves][BR], sl[kWaves][BR];

  const int Hkv = a.cache.kv_heads, h = blockIdx.x % Hkv, item = blockIdx.x / Hkv;
  const Partition<BR> part(a, blocks_bound);
  int b, local;
  if (!find_item(a.batch.batch, item, [&](int i) { return part.items(i); }, &b, &local)) return;
  const Seq s = sequence(a.batch, b);
  const int splits = part.splits(s), G = part.G;
  const Block blk = part.block(s, local / splits);
  const int T0 = blk.lo / kTile + local % splits * part.chunk;
  const int T1 = min((max(blk.hi, blk.lo) + kTile - 1) / kTile, splits > 1 ? T0 + part.chunk : 1 << 24);

  const int lane = __lane_id(), w = threadIdx.x / kWave, c = lane & 15, q = lane >> 4;
  const int P = a.cache.page_size, logP = __builtin_ctz(P);
  const uint8_t* const kc = static_cast<const uint8_t*>(a.cache.k);
  const uint8_t* const vc = static_cast<const uint8_t*>(a.cache.v);

  // query rows: lane (c, q) holds elements 64 piece + 16 q + 0 .. 15 of row c
  bf16x8 qf[NT][KK];
  int lo[NT], hi[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = blk.r0 + 16 * n + c;
    const bool valid = r < blk.rows;
    row_range(a, s, r, G, &lo[n], &hi[n]);
    if (!valid) hi[n] = 0;
    const uint16_t* src = static_cast<const uint16_t*>(a.q) + int64_t(s.start + r / G) * a.q_stride +
                          (h * G + r % G) * D + 16 * q;
#pragma unroll
    for (int k = 0; k < KK; ++k)
      qf[n][k] = valid ? *reinterpret_cast<const bf16x8*>(src + 64 * (k / 2) + 8 * (k % 2)) : bf16x8{};
  }

  f32x4 o[NT][DT];
  float m[NT], l[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m[n] = -INFINITY, l[n] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[n][d] = f32x4{};
  }

  // pages of the lane's key block (c / 4) and value block (q) in a tile
  auto page = [&](int tile, int blk16) {
    const int tok = tile * kTile + 16 * blk16;
    return tile < T1 && tok < s.kv ? page_of(a.batch, a.cache.pages, b, tok >> logP) : -1;
  };
  int kp = page(T0 + w, c >> 2), vp = page(T0 + w, q);
  for (int tile = T0 + w; tile < T1; tile += kWaves) {
    const bool kin = kp >= 0, vin = vp >= 0;
    const int64_t kh = int64_t(kin ? kp : 0) * Hkv + h, vh = int64_t(vin ? vp : 0) * Hkv + h;
    const uint8_t* kb = kc + kh * (P * D) + ((tile * kTile + 16 * (c >> 2)) & (P - 1)) * D + (c & 3) * D + 16 * q;
    const uint8_t* vb = vc + vh * (P * D) + c * P + ((tile * kTile + 16 * q) & (P - 1));
    u32x4 kx[4][kPieces], vx[DT];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < kPieces; ++i) kx[t][i] = *reinterpret_cast<const u32x4*>(kb + 4 * t * D + 64 * i);
    const float ks = a.cache.k_scale[kh], vs = vin ? a.cache.v_scale[vh] : 1.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) vx[d] = *reinterpret_cast<const u32x4*>(vb + 16 * d * P);
    kp = page(tile + kWaves, c >> 2), vp = page(tile + kWaves, q);

    f32x4 sc[NT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int n = 0; n < NT; ++n) sc[n][t] = f32x4{};
#pragma unroll
      for (int k = 0; k < KK; ++k) {
        const u32x4 u = kx[t][k / 2];
        const bf16x8 f = k % 2 ? decode8(u[2], u[3], ks) : decode8(u[0], u[1], ks);
#pragma unroll
        for (int n = 0; n < NT; ++n) sc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, qf[n][k], sc[n][t], 0, 0, 0);
      }
    }
    // what lies behind the sequence's last token may be any bytes: as values
    // they must be zeros (a probability of zero times NaN is NaN)
    const int first = tile * kTile + 16 * q;
    if (tile * kTile + kTile > s.kv || !__all(vin)) {
      const int count = vin ? min(max(s.kv - first, 0), 16) : 0;
#pragma unroll
      for (int d = 0; d < DT; ++d) vx[d] = first_codes(vx[d], count);
    }
    const bool masked = tile * kTile < blk.full_lo || tile * kTile + kTile > blk.full_hi || !__all(vin);
    bf16x8 p[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = sc[n][t][i] * a.scale2;
          if (masked) {
            const int j = first + 4 * t + i;
            x = vin && j >= lo[n] && j < hi[n] ? x : -INFINITY;
          }
          sc[n][t][i] = x;
          top = fmaxf(top, x);
        }
      {
        const auto u = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1]));
        const auto v = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1]));
      }
      const float mx = fmaxf(m[n], top), use = mx == -INFINITY ? 0.f : mx;
      if (__any(mx > m[n])) {
        const float f = __builtin_amdgcn_exp2f(m[n] - use);
        l[n] *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][d][i] *= f;
      }
      m[n] = mx;
      // each probability is rounded to bf16 once, for the product with values
      // that bf16 holds exactly; the sum takes it unrounded
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f(sc[n][t][i] - use);
          l[n] += e;
          p[n][t / 2][4 * (t % 2) + i] = __bf16(e);
        }
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const bf16x8 v0 = decode8(vx[d][0], vx[d][1], vs), v1 = decode8(vx[d][2], vx[d][3], vs);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, p[n][0], o[n][d], 0, 0, 0);
        o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, p[n][1], o[n][d], 0, 0, 0);
      }
    }
  }

  // join the waves
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    l[n] = row_sum4(l[n]);
    if (q == 0) sm[w][16 * n + c] = m[n], sl[w][16 * n + c] = l[n];
  }
  __syncthreads();
  float top[NT], f[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = 16 * n + c;
    top[n] = fmaxf(fmaxf(sm[0][r], sm[1][r]), fmaxf(sm[2][r], sm[3][r]));
    f[n] = m[n] == -INFINITY ? (l[n] == 0.f ? 0.f : l[n]) : __builtin_amdgcn_exp2f(m[n] - top[n]);
  }
  for (int turn = 0; turn < kWaves; ++turn) {
    if (turn == w) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          f32x4* at = reinterpret_cast<f32x4*>(so + (16 * n + c) * kLd + 16 * d + 4 * q);
          f32x4 x = turn ? *at : f32x4{};
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] += o[n][d][i] * f[n];
          *at = x;
        }
    }
    __syncthreads();
  }
  const int rows = min(BR, blk.rows - blk.r0);
  for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
    const int r = i / (D / 4), d = (i % (D / 4)) * 4;
    float mx = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) mx = fmaxf(mx, sm[k][r]);
#pragma unroll
    for (int k = 0; k < kWaves; ++k) sum += sm[k][r] == -INFINITY ? sl[k][r] : sl[k][r] * __builtin_amdgcn_exp2f(sm[k][r] - mx);
    const f32x4 x = *reinterpret_cast<const f32x4*>(so + r * kLd + d);
    if (splits > 1) {
      const int64_t slot = (int64_t(item) * Hkv + h) * BR + r;
      *reinterpret_cast<f32x4*>(a.part + slot * D + d) = x;
      if (d == 0) a.part_ml[2 * slot] = mx, a.part_ml[2 * slot + 1] = sum;
    } else {
      const int row = blk.r0 + r, t = s.start + row / G, head = h * G + row % G;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      uint16_t* dst = static_cast<uint16_t*>(a.out) + t * a.out_stride + head * D + d;
      *reinterpret_cast<u32x2*>(dst) = u32x2{to_bf16(x[0] * inv) | uint32_t(to_bf16(x[1] * inv)) << 16,
                                             to_bf16(x[2] * inv) | uint32_t(to_bf16(x[3] * inv)) << 16};
      if (a.lse && d == 0) a.lse[int64_t(t) * a.q_heads + head] = sum == 0.f ? -INFINITY : mx * kLn2 + logf(sum);
    }
  }
}

// The parts of a shared block added up in order: eight rows a workgroup.
template <int D, int BR>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, int blocks_bound) {
  constexpr int kLanes = D / 4, kRows = 256 / kLanes, kGroups = (BR + kRows - 1) / kRows;
  const int Hkv = a.cache.kv_heads, h = blockIdx.x % Hkv, at = blockIdx.x / Hkv, group = at % kGroups;
  const Partition<BR> part(a, blocks_bound);
  int b, k;
  if (!find_item(a.batch.batch, at / kGroups, [&](int i) { return part.blocks(sequence(a.batch, i)); }, &b, &k)) return;
  const Seq s = sequence(a.batch, b);
  const int splits = part.splits(s), G = part.G;
  if (splits == 1) return;  // written by its only item
  const int r = group * kRows + threadIdx.x / kLanes, d = (threadIdx.x % kLanes) * 4, row = k * BR + r;
  int base = 0;  // items of the sequences before b
  for (int b0 = 0; b0 < b; b0 += kWave) {
    const int i = b0 + __lane_id();
    base += wave_reduce_sum_i32(i < b ? part.items(i) : 0);
  }
  if (r >= BR || row >= part.rows(s)) return;
  const int64_t step = int64_t(Hkv) * BR, slot0 = (int64_t(base + k * splits) * Hkv + h) * BR + r;
  float mx = -INFINITY;
  for (int i = 0; i < splits; ++i) mx = fmaxf(mx, a.part_ml[2 * (slot0 + i * step)]);
  float sum = 0.f;
  f32x4 x{};
#pragma unroll 8
  for (int i = 0; i < splits; ++i) {
    const int64_t slot = slot0 + i * step;
    const float m = a.part_ml[2 * slot], l = a.part_ml[2 * slot + 1];
    const f32x4 y = *reinterpret_cast<const f32x4*>(a.part + slot * D + d);
    // a part without a score has a sum of 0, or of NaN if every score was
    const float f = m == -INFINITY ? l : __builtin_amdgcn_exp2f(m - mx);
    sum += m == -INFINITY ? l : l * f;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += f == 0.f ? 0.f : y[e] * f;
  }
  const int t = s.start + row / G, head = h * G + row % G;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  uint16_t* dst = static_cast<uint16_t*>(a.out) + t * a.out_stride + head * D + d;
  *reinterpret_cast<u32x2*>(dst) = u32x2{to_bf16(x[0] * inv) | uint32_t(to_bf16(x[1] * inv)) << 16,
                                         to_bf16(x[2] * inv) | uint32_t(to_bf16(x[3] * inv)) << 16};
  if (a.lse && d == 0) a.lse[int64_t(t) * a.q_heads + head] = sum == 0.f ? -INFINITY : mx * kLn2 + logf(sum);
}

template <int D, int BR>
hipError_t join(const AttendArgs& a, int blocks, hipStream_t s) {
  constexpr int kRows = 256 / (D / 4), kGroups = (BR + kRows - 1) / kRows;
  hipLaunchKernelGGL((k_attend_join<D, BR>), dim3(blocks * kGroups * a.cache.kv_heads), dim3(256), 0, s, a, blocks);
  return hipGetLastError();
}

}  // namespace

AttendPlan attend_plan(const wz_cache& c, const wz_ragged& r, int q_heads) {
  const int G = q_heads / c.kv_heads;
  const int64_t rows = int64_t(r.max_tokens) * G;
  AttendPlan p{};
  p.block_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  const int64_t each = (rows + p.block_rows - 1) / p.block_rows;
  const int64_t blocks = std::min({int64_t(r.batch) * each, int64_t(r.tokens) * G / p.block_rows + r.batch,
                                   int64_t(r.tokens) * G});
  p.blocks = int(std::min(blocks, int64_t(1) << 28));
  const int64_t tiles = (int64_t(r.max_kv) + 63) / 64;
  // items meant for the whole call: a few workgroups to a CU
  const int64_t meant = std::max<int64_t>(1, (p.block_rows > 64 ? 2 : 4) * kCUs / c.kv_heads);
  p.shared = tiles > 8 && p.blocks < meant;
  p.slots = p.blocks + (p.shared ? int(meant) : 0);
  if (p.shared) {
    const size_t n = size_t(p.slots) * c.kv_heads * p.block_rows;
    p.part_bytes = (n * c.head_dim * 4 + 255) / 256 * 256;
    p.ml_bytes = (n * 8 + 255) / 256 * 256;
    p.bytes = p.part_bytes + p.ml_bytes;
  }
  return p;
}

hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  const dim3 grid(p.slots * a.cache.kv_heads), block(kThreads);
  const int D = a.cache.head_dim;
  if (p.block_rows > 64) {
    const hipError_t e = launch_attend_prompt(a, p, s);
    if (e != hipSuccess) return e;
  } else if (D == 128) {
    if (p.block_rows == 16) hipLaunchKernelGGL((k_attend_token<128, 1>), grid, block, 0, s, a, p.blocks);
    else if (p.block_rows == 32) hipLaunchKernelGGL((k_attend_token<128, 2>), grid, block, 0, s, a, p.blocks);
    else hipLaunchKernelGGL((k_attend_token<128, 4>), grid, block, 0, s, a, p.blocks);
  } else {
    if (p.block_rows == 16) hipLaunchKernelGGL((k_attend_token<64, 1>), grid, block, 0, s, a, p.blocks);
    else if (p.block_rows == 32) hipLaunchKernelGGL((k_attend_token<64, 2>), grid, block, 0, s, a, p.blocks);
    else hipLaunchKernelGGL((k_attend_token<64, 4>), grid, block, 0, s, a, p.blocks);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.shared) return e;
  switch (p.block_rows) {
    case 16: return D == 128 ? join<128, 16>(a, p.blocks, s) : join<64, 16>(a, p.blocks, s);
    case 32: return D == 128 ? join<128, 32>(a, p.blocks, s) : join<64, 32>(a, p.blocks, s);
    case 64: return D == 128 ? join<128, 64>(a, p.blocks, s) : join<64, 64>(a, p.blocks, s);
    default: return D == 128 ? join<128, 128>(a, p.blocks, s) : join<64, 128>(a, p.blocks, s);
  }
}

}  // namespace wz
