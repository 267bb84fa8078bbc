// How the attention kernels share out a ragged batch: row blocks and, where
// there are few of them, runs of tokens of each block.
//
// The rows of sequence b under one key/value head are its new tokens times
// the head's group of query heads, token by token: row i * G + g.  They fall
// into blocks of BR rows.  A block's tokens are worked on in tiles of 64; in a
// shared plan a block's tiles are split into runs of `chunk` tiles, an item
// each, where chunk follows from the whole batch's tiles, so that a long
// sequence gets more workgroups than a short one and all finish together.
#pragma once

#include "wz_serve.h"

namespace wz {

constexpr int kTile = 64;       // tokens of a tile
constexpr int kMinChunk = 4;    // tiles: an item is at least this long where blocks are shared

struct Block {
  int rows, r0;            // rows of the sequence, first row of the block
  int lo, hi;              // places that any of its rows sees: [lo, hi)
  int full_lo, full_hi;    // places that every one of its rows sees
};

template <int BR>
struct Partition {
  const AttendArgs& a;
  int G, chunk;

  __device__ __forceinline__ int rows(const Seq& s) const { return s.n * G; }
  __device__ __forceinline__ int blocks(const Seq& s) const { return (rows(s) + BR - 1) / BR; }
  // tiles that a block of the sequence spans at most
  __device__ __forceinline__ int tiles(const Seq& s) const {
    const int all = (s.kv + kTile - 1) / kTile;
    if (!(a.causal && a.window > 0)) return all;
    const int64_t span = int64_t(a.window) + (BR - 1) / G + 1;
    return int(min(int64_t(all), (span + kTile - 1) / kTile + 1));
  }
  __device__ __forceinline__ int splits(const Seq& s) const {
    return a.shared ? max(1, (tiles(s) + chunk - 1) / chunk) : 1;
  }
  __device__ __forceinline__ int items(int b) const {
    const Seq s = sequence(a.batch, b);
    return blocks(s) * splits(s);
  }
  // The same in every workgroup: the tiles of all blocks over the items that
  // are meant for them; the host's bound on slots leaves one more a block.
  __device__ __forceinline__ Partition(const AttendArgs& args, int blocks_bound)
      : a(args), G(args.q_heads / args.cache.kv_heads), chunk(1 << 30) {
    if (!a.shared) return;
    double total = 0;
    for (int b0 = 0; b0 < a.batch.batch; b0 += kWave) {
      const int b = b0 + __lane_id();
      if (b < a.batch.batch) {
        const Seq s = sequence(a.batch, b);
        total += double(blocks(s)) * tiles(s);
      }
    }
    total = wave_reduce_f64(total, [](double x, double y) { return x + y; });
    const int meant = max(a.slots - blocks_bound, 1);
    const double c = ceil(total / meant);
    chunk = c < (1 << 24) ? max(int(c), kMinChunk) : (1 << 24);
  }
  __device__ __forceinline__ Block block(const Seq& s, int k) const {
    Block x;
    x.rows = rows(s);
    x.r0 = k * BR;
    const int first = s.place0 + x.r0 / G, last = s.place0 + (min(x.r0 + BR, x.rows) - 1) / G;
    x.hi = a.causal ? min(last + 1, s.kv) : s.kv;
    x.full_hi = a.causal ? min(first + 1, s.kv) : s.kv;
    x.lo = a.causal && a.window > 0 ? max(0, first - a.window + 1) : 0;
    x.full_lo = a.causal && a.window > 0 ? max(0, last - a.window + 1) : 0;
    return x;
  }
};

// The places [lo, hi) that row r of a sequence sees.
__device__ __forceinline__ void row_range(const AttendArgs& a, const Seq& s, int r, int G, int* lo, int* hi) {
  const int place = s.place0 + r / G;
  *hi = a.causal ? min(place + 1, s.kv) : s.kv;
  *lo = a.causal && a.window > 0 ? max(0, place - a.window + 1) : 0;
}

// Eight codes (two words) as bf16 numbers times a power of two: exact.
__device__ __forceinline__ bf16x8 decode8(uint32_t a, uint32_t b, float scale) {
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  const v2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
  const v2 y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
  const v2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
  const v2 w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  return bf16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

// The first `count` of 16 codes, zeros for the rest.
__device__ __forceinline__ u32x4 first_codes(u32x4 v, int count) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = count - 4 * i;
    v[i] = c >= 4 ? v[i] : c <= 0 ? 0u : v[i] & ((1u << (8 * c)) - 1u);
  }
  return v;
}

__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, __bf16(x)); }

constexpr float kLn2 = 0.69314718055994531f;

}  // namespace wz
