// How the attention kernels share out a ragged batch.
//
// The rows of sequence b under one key/value head are its new tokens times
// the head's group of query heads, token by token: row i * G + g.  They fall
// into blocks of BR rows; a block's tokens are worked on in tiles of 64.
//
// Where blocks are few or long they are shared: all blocks' tiles, one block
// behind the other, are cut into equal runs, one for each workgroup (for
// each key/value head), so that a long sequence gets more workgroups than a
// short one and all finish together.  A workgroup leaves a part of every
// block that it does not have to itself in slot (its number + the block's),
// and a second kernel adds a block's parts up in order.
//
// Few rows in few blocks are cut so that no workgroup has tiles of two blocks,
// since a piece of a block costs as much as a round of tiles: each block into
// equal pieces of `run` tiles or fewer, one for each workgroup, whose number is
// the piece's slot.
#pragma once

#include "wz_serve.h"

namespace wz {

constexpr int kTile = 64;       // tokens of a tile
constexpr int kMinRun = 4;      // tiles of a workgroup's run at least
constexpr int kStartTiles = 3;  // few rows: what beginning a block counts as

// Whether blocks are cut by themselves, and the tiles of their pieces at most: the
// pieces, total / run and one more for each block at most, must not outnumber
// the workgroups.
__host__ __device__ inline bool lone_pieces(int64_t blocks, int workers) { return 4 * blocks <= workers; }
__host__ __device__ inline int64_t lone_run(int64_t total, int64_t blocks, int workers) {
  const int64_t run = (total + workers - blocks - 1) / (workers - blocks);
  return run > kMinRun ? run : kMinRun;
}

struct Block {
  int rows, r0;            // rows of the sequence, first row of the block
  int lo, hi;              // places that any of its rows sees: [lo, hi)
  int full_lo, full_hi;    // places that every one of its rows sees
};

// A place in the shared plan: tile `off` of the `tiles` that block k of
// sequence seq has; `block` blocks and `before` tiles lie in front of that one.
// (Where blocks are cut by themselves, pieces take the place of tiles.)
struct Spot {
  int seq, k, off, tiles, block, before;
  Seq s;
};

template <int BR>
struct Partition {
  const AttendArgs& a;
  int G;
  int total, run;  // shared: tiles of all blocks, and of a workgroup's run
  bool lone;       // shared: blocks are cut by themselves

  __device__ __forceinline__ int blocks(const Seq& s) const { return (s.n * G + BR - 1) / BR; }
  __device__ __forceinline__ Block block(const Seq& s, int k) const {
    Block x;
    x.rows = s.n * G;
    x.r0 = k * BR;
    const int first = s.place0 + x.r0 / G, last = s.place0 + (min(x.r0 + BR, x.rows) - 1) / G;
    x.hi = a.causal ? min(last + 1, s.kv) : s.kv;
    x.full_hi = a.causal ? min(first + 1, s.kv) : s.kv;
    x.lo = a.causal && a.window > 0 ? max(0, first - a.window + 1) : 0;
    x.full_lo = a.causal && a.window > 0 ? max(0, last - a.window + 1) : 0;
    return x;
  }
  // The tiles of a block: one if it sees nothing, since its rows have to be
  // written.  With few rows to a block (the token kernel) all blocks of a
  // sequence count as many as the widest may span, so that the sequence's sum
  // is a product.
  static constexpr bool kUniform = BR <= 64;
  // A block counts as kStart tiles more than it has, at its front: what a
  // workgroup loses when it begins one (next tokens of 64 sequences of 500 to
  // 8 200 tokens 54.3 us without, 51.9, 51.5 and 51.3 with 2, 3 and 5; of 64 others
  // 41.4, 41.0, 37.9 and 37.4; but few rows of 12 long sequences 94, 94, 93 and 99).
  static constexpr int kStart = kUniform ? kStartTiles : 0;
  __device__ __forceinline__ int tiles(const Seq& s, int k) const {
    if constexpr (kUniform) {
      const int all = max(1, (s.kv + kTile - 1) / kTile);
      if (!(a.causal && a.window > 0)) return all;
      const int64_t span = int64_t(a.window) + (BR - 1) / G + 1;
      return int(min(int64_t(all), (span + kTile - 1) / kTile + 1));
    } else {
      const Block x = block(s, k);
      return max(1, (x.hi + kTile - 1) / kTile - x.lo / kTile);
    }
  }
  // The first block whose running count of blocks (TILES: of tiles) passes
  // `at`; false if none does, with the counts of all blocks.
  template <bool TILES>
  __device__ __forceinline__ bool find(int at, Spot* spot) const {
    const int lane = __lane_id();
    int nb = 0, nt = 0;
    for (int b0 = 0; b0 < a.batch.batch; b0 += kWave) {
      const bool in = b0 + lane < a.batch.batch;
      const Seq s = in ? sequence(a.batch, b0 + lane) : Seq{0, 0, 0, 0};
      const int mine = blocks(s);
      if constexpr (kUniform) {
        const int all = tiles(s, 0), each = lone ? (all + run - 1) / run : all + kStart;
        const int work = a.shared ? mine * each : 0;  // (unshared, tiles are not asked for)
        const int ib = wave_incl_scan_i32(mine), it = wave_incl_scan_i32(work);
        const unsigned long long pass = __ballot(TILES ? nt + it > at : nb + ib > at);
        if (pass) {
          const int l = __builtin_ctzll(pass);
          const int b1 = nb + __builtin_amdgcn_readlane(ib - mine, l);
          const int t1 = nt + __builtin_amdgcn_readlane(it - work, l);
          const int n = __builtin_amdgcn_readlane(each, l);
          const int k = TILES ? (at - t1) / n : at - b1;
          *spot = Spot{b0 + l, k, TILES ? (at - t1) % n : 0, n, b1 + k, t1 + k * n, sequence_of_lane(s, l)};
          return true;
        }
        nb += __builtin_amdgcn_readlane(ib, kWave - 1), nt += __builtin_amdgcn_readlane(it, kWave - 1);
      } else {
        for (unsigned long long left = __ballot(mine > 0); left; left &= left - 1) {
          const int l = __builtin_ctzll(left);
          const Seq one = sequence_of_lane(s, l);
          const int count = blocks(one);
          if (!TILES && at >= nb + count && !a.shared) {  // (tiles are not needed)
            nb += count;
            continue;
          }
          for (int k0 = 0; k0 < count; k0 += kWave) {
            const int n = k0 + lane < count ? tiles(one, k0 + lane) : 0;
            const int it = wave_incl_scan_i32(n);
            const unsigned long long pass = __ballot(n > 0 && (TILES ? nt + it > at : nb + k0 + lane + 1 > at));
            if (pass) {
              const int i = __builtin_ctzll(pass), t1 = nt + __builtin_amdgcn_readlane(it - n, i);
              *spot = Spot{b0 + l, k0 + i, TILES ? at - t1 : 0, __builtin_amdgcn_readlane(n, i), nb + k0 + i, t1, one};
              return true;
            }
            nt += __builtin_amdgcn_readlane(it, kWave - 1);
          }
          nb += count;
        }
      }
    }
    spot->block = nb, spot->before = nt;
    return false;
  }
  // (the host shares only where the tiles of all blocks fit in an int)
  __device__ __forceinline__ Partition(const AttendArgs& args)
      : a(args), G(args.q_heads / args.cache.kv_heads), total(0), run(0), lone(false) {
    if (!a.shared) return;
    Spot all;
    find<true>(0x7fffffff, &all);
    total = all.before;
    run = max((total + a.workers - 1) / a.workers, kMinRun);
    if (kUniform && lone_pieces(all.block, a.workers)) {
      run = int(lone_run(total, all.block, a.workers));
      lone = true;
    }
  }
  // Calls f(spot, count, slot) for every piece of a block that workgroup `me`
  // has: `count` tiles from the spot on; slot is where its part goes, -1 if the
  // block is all its own.
  template <typename F>
  __device__ __forceinline__ void each_piece(int me, F f) const {
    Spot x;
    if (!a.shared) {
      if (find<false>(me, &x)) f(x, x.tiles, -1);
      return;
    }
    if (lone) {
      if (!find<true>(me, &x) || x.block >= a.blocks) return;
      const int all = tiles(x.s, 0), from = all * x.off / x.tiles, to = all * (x.off + 1) / x.tiles;
      const int slot = x.tiles == 1 ? -1 : me;
      x.off = from;
      f(x, to - from, slot);
      return;
    }
    int at = me * run;
    const int end = min(at + run, total);
    // (rows that overlap, against the contract, may make more blocks than the
    // workspace has slots for)
    while (at < end && find<true>(at, &x) && x.block < a.blocks) {
      const int count = min(end - at, x.tiles - x.off), slot = count == x.tiles ? -1 : me + x.block;
      const int to = max(x.off + count - kStart, 0);
      at += count;
      x.off = max(x.off - kStart, 0);
      f(x, to - x.off, slot);
      if (at < end) __syncthreads();  // LDS is used again
    }
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
