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
// The waves take a block's tiles in turn, each with a running maximum and sum,
// and join through LDS at the end in a fixed order.
//
// Measured: next tokens of four sequences of 60 000 to 131 000 tokens, 28 heads of
// 128 over 4, 349 MB in 64.6 us and 5 us for the join (a 1 GiB copy's 5.2 TB/s
// would take 66.8); of 64 sequences of 500 to 8 200, 212 MB in 46 and 5.
#include "wz_attend.h"

namespace wz {
namespace {

// `count` tiles from spot x on, key/value head h; slot: where their part goes, -1
// if the block is this workgroup's alone.
//
// Four waves take a block's tiles: with eight, next tokens of 1 to 64 sequences and
// four heads, 128 to 1536 tokens, one workgroup to a block, took 6.7 to 23.3 us
// where four took 6.1 to 21.7 (heads of 64 elements: 5.5 to 13.6 and 5.2 to 12.8).
constexpr int kWaves = 4;
template <int D, int NT>
__device__ __forceinline__ void attend_block(const AttendArgs& a, const Partition<16 * NT>& part, int h, const Spot& x,
                                             int count, int slot, float* so, float (*sm)[16 * NT],
                                             float (*sl)[16 * NT]) {
  constexpr int BR = 16 * NT, KK = D / 32, DT = D / 16, kPieces = D / 64, kThreads = kWaves * kWave;
  constexpr int kLd = D + 4;
  const int Hkv = a.cache.kv_heads, G = part.G;
  const Seq s = x.s;
  const Block blk = part.block(s, x.k);
  const int T0 = blk.lo / kTile + x.off;
  const int T1 = min((max(blk.hi, blk.lo) + kTile - 1) / kTile, T0 + count);

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

  // Codes of a tile as they come, two tiles to a wave: the loads of the next
  // one are under way while this one is worked on.  Nothing branches around a
  // load: what lies behind the last tile is the last tile again, and a block
  // that has no page reads page 0 and is masked.
  struct Tile {
    u32x4 kx[4][kPieces], vx[DT];
    float ks, vs;
    bool vin;
  } bufs[2];
  const int last = T0 + w + (max(T1 - T0 - w, 1) - 1) / kWaves * kWaves;  // this wave's last tile
  const int* const row = a.batch.table + int64_t(x.seq) * a.batch.table_stride;
  const int entries = max((s.kv + P - 1) >> logP, 1);
  // Pages of the lane's key block (c / 4) and value block (q) in a tile: asked
  // for before the loads of the tile in front, so that waiting for them does
  // not wait for those.
  struct Pages {
    int k, v;
  } ids[2];
  auto pages = [&](int tile) {
    const int tok = min(tile, last) * kTile;
    return Pages{row[min((tok + 16 * (c >> 2)) >> logP, entries - 1)], row[min((tok + 16 * q) >> logP, entries - 1)]};
  };
  auto load = [&](Tile& x, int tile, Pages id) {
    const int tok = min(tile, last) * kTile, kp = id.k, vp = id.v;
    const bool kin = uint32_t(kp) < uint32_t(a.cache.pages);
    x.vin = uint32_t(vp) < uint32_t(a.cache.pages);
    const int64_t kh = int64_t(kin ? kp : 0) * Hkv + h, vh = int64_t(x.vin ? vp : 0) * Hkv + h;
    const uint8_t* kb = kc + kh * (P * D) + ((tok + 16 * (c >> 2)) & (P - 1)) * D + (c & 3) * D + 16 * q;
    const uint8_t* vb = vc + vh * (P * D) + c * P + ((tok + 16 * q) & (P - 1));
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < kPieces; ++i) x.kx[t][i] = *reinterpret_cast<const u32x4*>(kb + 4 * t * D + 64 * i);
    x.ks = a.cache.k_scale[kh], x.vs = a.cache.v_scale[vh];
#pragma unroll
    for (int d = 0; d < DT; ++d) x.vx[d] = *reinterpret_cast<const u32x4*>(vb + 16 * d * P);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto work = [&](Tile& x, int tile) {
    const bool vin = x.vin;
    const float ks = x.ks, vs = vin ? x.vs : 1.f;
    u32x4 (&kx)[4][kPieces] = x.kx, (&vx)[DT] = x.vx;
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
#pragma unroll
      for (int t = 0; t < 4; ++t) sc[n][t] *= a.scale2;
      if (masked) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = first + 4 * t + i;
            sc[n][t][i] = vin && j >= lo[n] && j < hi[n] ? sc[n][t][i] : -INFINITY;
          }
      }
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[n][t][i]);
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
      // that bf16 holds exactly, on the matrix cores' rate for bf16; the sum takes
      // it unrounded, so a row's weights add up to one within 2^-9 (error against
      // 64 bits, of results in bf16: 0.0016 to 0.0017, with fp32 probabilities 0.0016)
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
  };
  if (T0 + w < T1) {
    ids[0] = pages(T0 + w);
    ids[1] = pages(T0 + w + kWaves);
    load(bufs[0], T0 + w, ids[0]);
    for (int tile = T0 + w; tile < T1; tile += 2 * kWaves) {
      ids[0] = pages(tile + 2 * kWaves);
      load(bufs[1], tile + kWaves, ids[1]);
      work(bufs[0], tile);
      if (tile + kWaves >= T1) break;
      ids[1] = pages(tile + 3 * kWaves);
      load(bufs[0], tile + 2 * kWaves, ids[0]);
      work(bufs[1], tile + kWaves);
    }
  }

  // join the waves
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    l[n] = row_sum4(l[n]);
    if (q == 0) sm[w][16 * n + c] = m[n], sl[w][16 * n + c] = l[n];
  }
  __syncthreads();
  float f[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = fmaxf(top, sm[i][16 * n + c]);
    // a wave without a score has a sum of 0, or of NaN if every score was
    f[n] = m[n] == -INFINITY ? l[n] : __builtin_amdgcn_exp2f(m[n] - top);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      f32x4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = o[n][d][i] * f[n];
      *reinterpret_cast<f32x4*>(so + (w * BR + 16 * n + c) * kLd + 16 * d + 4 * q) = x;
    }
  }
  __syncthreads();
  const int rows = min(BR, blk.rows - blk.r0);
  for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
    const int r = i / (D / 4), d = (i % (D / 4)) * 4;
    float mx = -INFINITY, sum = 0.f;
    f32x4 x{};
#pragma unroll
    for (int u = 0; u < kWaves; ++u) mx = fmaxf(mx, sm[u][r]);
#pragma unroll
    for (int u = 0; u < kWaves; ++u) {
      sum += sm[u][r] == -INFINITY ? sl[u][r] : sl[u][r] * __builtin_amdgcn_exp2f(sm[u][r] - mx);
      x += *reinterpret_cast<const f32x4*>(so + (u * BR + r) * kLd + d);
    }
    if (slot >= 0) {
      const int64_t at = (int64_t(slot) * Hkv + h) * BR + r;
      *reinterpret_cast<f32x4*>(a.part + at * D + d) = x;
      if (d == 0) a.part_ml[2 * at] = mx, a.part_ml[2 * at + 1] = sum;
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

template <int D, int NT>
__global__ __launch_bounds__(kWaves* kWave, NT == 1 ? 2 : 1) void k_attend_token(AttendArgs a) {
  constexpr int BR = 16 * NT;
  __shared__ __align__(16) float so[kWaves * BR * (D + 4)];
  __shared__ float sm[kWaves][BR], sl[kWaves][BR];
  const int Hkv = a.cache.kv_heads, h = blockIdx.x % Hkv, me = blockIdx.x / Hkv;
  const Partition<BR> part(a);
  part.each_piece(me, [&](const Spot& x, int count, int slot) {
    attend_block<D, NT>(a, part, h, x, count, slot, so, sm, sl);
  });
}

// The parts of a shared block added up.  A workgroup has 256 / (D / 4) groups
// of lanes; PG of them share a row, taking its parts in turn, so that a row of
// many parts costs a few loads' latency, and add up through LDS in order.
template <int D, int BR, int PG>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a) {
  constexpr int kLanes = D / 4, kRows = 256 / kLanes / PG;  // rows of a workgroup
  __shared__ __align__(16) float sums[256 / kLanes][D];
  __shared__ float red[2][256 / kLanes];
  const int Hkv = a.cache.kv_heads, h = blockIdx.x % Hkv, at = blockIdx.x / Hkv;
  const Partition<BR> part(a);
  const int per = (a.block_rows + kRows - 1) / kRows;  // workgroups of a block
  Spot x;
  if (!part.template find<false>(at / per, &x)) return;
  const Seq s = x.s;
  const int first = part.lone ? x.before : x.before / part.run;
  const int last = part.lone ? x.before + x.tiles - 1 : (x.before + x.tiles - 1) / part.run;
  if (first == last) return;  // written by the only workgroup that had it
  const int lane = threadIdx.x % kLanes, all_groups = threadIdx.x / kLanes, d = 4 * lane;
  const int group = all_groups % PG, mine = all_groups / PG;
  const int G = part.G, r = at % per * kRows + mine, row = x.k * BR + r;
  const bool in = row < s.n * G;  // (its slots exist in any case)
  const int64_t step = int64_t(Hkv) * BR, slot0 = (int64_t(first + (part.lone ? 0 : x.block)) * Hkv + h) * BR + r;
  // a running maximum as in the kernels that left the parts; a part without a
  // score has a maximum of -inf and a sum of 0, or of NaN if every score was
  float top = -INFINITY, sum = 0.f;
  f32x4 o{};
  for (int i = first + group; i <= last; i += 4 * PG) {
    float m[4], l[4];
    f32x4 y[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {  // four parts at once; behind the last one the first again, without weight
      const int j = i + u * PG;
      const int64_t slot = slot0 + (j <= last ? j - first : 0) * step;
      m[u] = a.part_ml[2 * slot], l[u] = a.part_ml[2 * slot + 1];
      y[u] = *reinterpret_cast<const f32x4*>(a.part + slot * D + d);
      if (j > last) m[u] = -INFINITY, l[u] = 0.f;
    }
    float next = top;
#pragma unroll
    for (int u = 0; u < 4; ++u) next = fmaxf(next, m[u]);
    const float use = next == -INFINITY ? 0.f : next, keep = __builtin_amdgcn_exp2f(top - use);
    sum *= keep;
    o *= keep;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float f = m[u] == -INFINITY ? l[u] : __builtin_amdgcn_exp2f(m[u] - use);
      sum += m[u] == -INFINITY ? l[u] : l[u] * f;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += f == 0.f ? 0.f : y[u][e] * f;
    }
    top = next;
  }
  float mx = top, total = sum;
  if constexpr (PG > 1) {
    if (lane == 0) red[0][all_groups] = top, red[1][all_groups] = sum;
    __syncthreads();
    const float *const tops = red[0] + mine * PG, *const sum_of = red[1] + mine * PG;
    total = 0.f;
#pragma unroll
    for (int i = 0; i < PG; ++i) mx = fmaxf(mx, tops[i]);
#pragma unroll
    for (int i = 0; i < PG; ++i)
      total += tops[i] == -INFINITY ? sum_of[i] : sum_of[i] * __builtin_amdgcn_exp2f(tops[i] - mx);
    *reinterpret_cast<f32x4*>(sums[all_groups] + d) = o * (top == -INFINITY ? sum : __builtin_amdgcn_exp2f(top - mx));
    __syncthreads();
    if (group > 0) return;
    o = f32x4{};
#pragma unroll
    for (int i = 0; i < PG; ++i) o += *reinterpret_cast<const f32x4*>(sums[mine * PG + i] + d);
  }
  if (!in) return;
  const int t = s.start + row / G, head = h * G + row % G;
  const float inv = total == 0.f ? 0.f : 1.f / total;
  uint16_t* dst = static_cast<uint16_t*>(a.out) + t * a.out_stride + head * D + d;
  *reinterpret_cast<u32x2*>(dst) = u32x2{to_bf16(o[0] * inv) | uint32_t(to_bf16(o[1] * inv)) << 16,
                                         to_bf16(o[2] * inv) | uint32_t(to_bf16(o[3] * inv)) << 16};
  if (a.lse && d == 0) a.lse[int64_t(t) * a.q_heads + head] = total == 0.f ? -INFINITY : mx * kLn2 + logf(total);
}

template <int D, int BR>
hipError_t join(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  // groups share rows where blocks have eight parts or more on average (next
  // tokens of four heads over 30 000 tokens, shared and not: one sequence 19 and 34
  // us, four 31 and 34, twelve 78 and 78, 24 143 and 141; 36 rows over 8000 33 and
  // 36, 150 rows 55 and 45)
  constexpr int kGroups = 1024 / D;
  const bool many = p.workers >= 8 * p.blocks;
  const int rows = many ? 1 : kGroups;  // of a workgroup
  const dim3 grid(uint32_t(p.blocks * ((a.block_rows + rows - 1) / rows) * a.cache.kv_heads)), block(256);
  if (many) hipLaunchKernelGGL((k_attend_join<D, BR, kGroups>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_attend_join<D, BR, 1>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <int D>
void launch_token(const AttendArgs& a, const AttendPlan& p, int64_t groups, hipStream_t s) {
  const dim3 grid{uint32_t(groups)}, block{kWaves * kWave};
  if constexpr (D == 64)
    if (p.block_rows == 64) {
      hipLaunchKernelGGL((k_attend_token<D, 4>), grid, block, 0, s, a);
      return;
    }
  if (p.block_rows == 32) hipLaunchKernelGGL((k_attend_token<D, 2>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_attend_token<D, 1>), grid, block, 0, s, a);
}

}  // namespace

AttendPlan attend_plan(const wz_cache& c, const wz_ragged& r, int q_heads, int window) {
  const int G = q_heads / c.kv_heads;
  const int64_t rows = int64_t(r.max_tokens) * G;
  AttendPlan p{};
  auto blocks = [&](int br) {
    const int64_t each = (rows + br - 1) / br;
    return std::min({int64_t(r.batch) * each, int64_t(r.tokens) * G / br + r.batch, int64_t(r.tokens) * G});
  };
  // (64 rows of 128 elements would not fit a wave's registers: two blocks of 32
  // read the keys twice, the second time from L2: 35 rows each of 32 sequences of
  // 950 tokens 19 us, as blocks of 64 46 and of 128 26)
  p.block_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? (c.head_dim == 64 ? 64 : 32) : 128;
  p.blocks = int(std::min(blocks(p.block_rows), int64_t(1) << 28));
  int64_t tiles = (int64_t(r.max_kv) + kTile - 1) / kTile;
  if (window > 0) tiles = std::min(tiles, (int64_t(window) + (p.block_rows - 1) / G + kTile) / kTile + 1);
  // A CU runs two workgroups of four waves at once, or one of those whose waves
  // take more than half the registers (with two planned for, 28 rows each of 10
  // sequences of 2000 tokens took 30 us instead of 20), or one prompt workgroup of
  // eight.  Registers would hold four of few rows: more parts, shorter runs, and
  // 74 us instead of 70 for the next tokens of four sequences of 60 000 to 131 000
  // (three: 72; of 64 of 500 to 8 200: 55 with two, 63, 54).
  // Eight waves to a prompt's workgroup: a prompt of 28 heads over 4, with four
  // waves and with eight, of 100 rows (24 blocks times heads) 11.6 and 13.1 us, 800
  // (176) 24.4 and 23.0, 1286 (284) 35.2 and 31.4, 1400 (308) 37.4 and 33.1, 2000
  // (440) 51 and 50, 2600 (572) 70 and 78.  Equal blocks lose as soon as they need
  // a second round: 128 rows each of 60 sequences, 500 tokens before them, 4 heads
  // (240) 29.3 and 28.6, of 80 (320) 33.5 and 43.2, of 100 (400) 36.7 and 48.2.
  p.groups = int64_t(p.blocks) * c.kv_heads <= kCUs * 5 / 4 ? 2 : 1;
  const bool wide = p.block_rows == 64 || (p.block_rows == 32 && c.head_dim == 128);
  const int at_once = wide || (p.block_rows == 128 && p.groups == 2) ? kCUs : 2 * kCUs;
  p.workers = int(std::max(1, at_once / c.kv_heads));
  // Few rows in few blocks: sharing costs a second launch, which is worth four of
  // the rounds that four waves make over a block's tiles where it has 16 rows (as
  // the rule counts them, two of eight tiles), and two where it has more.  Not
  // shared and shared, one to four sequences of four heads of 128:
  //   7 rows    1024 tokens 11.2 and 12.2 us, 1280 12.5 and 12.3, 1536 13.9 and 12.7
  //   25 rows   512 tokens 12.5 and 15.7, 768 14.6 and 15.9, 1024 16.4 and 15.9
  // (heads of 64 cross later: 7.8 and 10.6 at 1024 tokens, 10.7 and 10.8 at 2048.)
  // Prompts: a block alone takes as many turns as it has tiles, a shared run its
  // share of all tiles, and the parts, their join and what begins a piece come to
  // 24 turns (28 heads of 128 over 4, not shared and shared: 100 rows over 1500
  // tokens 32 and 36 us, over 2000 40 and 37, over 5000 78 and 42; a prompt of 1600
  // 41 and 89, of 2200 56 and 113; 1000 rows over 4000 tokens 81 and 100; 300 over
  // 6000 94 and 56; 400 over 16000 226 and 119).
  // Few rows in more blocks: sharing makes up for unequal lengths, which the
  // bounds do not tell.  64 sequences of four heads, not shared and shared: 1536
  // tokens each 21.7 and 28.3 us, 4096 each 53 and 63, 64 to 4096 31 and 34; one of
  // 1280 beside others of 191 14.5 and 17.1, one of 2048 19.2 and 17.9, one of 4096
  // 29 and 19; 128 sequences of 100 to 8000 102 and 75.
  bool long_enough = tiles > 24 + (p.block_rows > 64 ? p.blocks * tiles / p.workers : 0);
  if (p.block_rows <= 64 && lone_pieces(p.blocks, p.workers)) {
    const int64_t run = lone_run(p.blocks * tiles, p.blocks, p.workers);
    const int round = p.block_rows == 16 ? 8 : 4;
    long_enough = (tiles + round - 1) / round >= (run + 3) / 4 + 2;
  }
  // Many blocks level out by themselves unless one is far longer than the others
  // (next tokens of four heads, not shared and shared; 256 sequences: 2000 tokens
  // each 101 and 112 us, 100 to 8000 126 and 121, one of 60 000 beside others of
  // 200 324 and 53; 512 sequences: 189 and 219, 198 and 226, 339 and 94).
  // (every sequence at its bounds, so that no array's contents make the tiles pass 32 bits)
  const int64_t most = int64_t(r.batch) * ((rows + p.block_rows - 1) / p.block_rows) * (tiles + 1 + kStartTiles);
  p.shared = long_enough && most < (int64_t(1) << 30) &&
             (p.block_rows > 64 ? p.blocks < p.workers : int64_t(p.blocks) * c.kv_heads < 2048);
  p.slots = p.blocks + p.workers;
  if (p.shared) {
    const size_t n = size_t(p.slots) * c.kv_heads * p.block_rows;
    p.part_bytes = (n * c.head_dim * 4 + 255) / 256 * 256;
    p.ml_bytes = (n * 8 + 255) / 256 * 256;
    p.bytes = p.part_bytes + p.ml_bytes;
  }
  return p;
}

hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  const int64_t groups = int64_t(p.shared ? p.workers : p.blocks) * a.cache.kv_heads;
  const int D = a.cache.head_dim;
  if (p.block_rows > 64) {
    const hipError_t e = launch_attend_prompt(a, p, s);
    if (e != hipSuccess) return e;
  } else if (D == 128) {
    launch_token<128>(a, p, groups, s);
  } else {
    launch_token<64>(a, p, groups, s);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.shared) return e;
  switch (p.block_rows) {
    case 16: return D == 128 ? join<128, 16>(a, p, s) : join<64, 16>(a, p, s);
    case 32: return D == 128 ? join<128, 32>(a, p, s) : join<64, 32>(a, p, s);
    case 64: return join<64, 64>(a, p, s);
    default: return D == 128 ? join<128, 128>(a, p, s) : join<64, 128>(a, p, s);
  }
}

}  // namespace wz
