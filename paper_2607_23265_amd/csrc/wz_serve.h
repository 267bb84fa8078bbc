// Shared by the serving operators (include/wavezip_serve.h): the cache's
// codes, the ragged batch on the device, and the launchers.
#pragma once

#include "wavezip_serve.h"
#include "wz_device.h"

namespace wz {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kE4m3Max = 448.f;
constexpr int kScaleMinExp = -100, kScaleMaxExp = 119;

// Sequence b of a ragged batch with every value cut to the ranges the host
// checked, so that nothing below reads outside the arrays whatever they hold.
struct Seq {
  int start, n;   // first row and number of new tokens (at most max_tokens)
  int kv;         // tokens in the cache, these counted
  int place0;     // place of the first new token (negative if n > kv)
};
__device__ __forceinline__ Seq sequence(const wz_ragged& r, int b) {
  Seq s;
  s.start = min(max(r.start[b], 0), r.tokens);
  const int all = max(min(r.start[b + 1], r.tokens) - s.start, 0);
  s.kv = min(max(r.kv_len[b], 0), r.max_kv);
  s.place0 = s.kv - all;
  s.n = min(all, r.max_tokens);
  return s;
}

// Lane l's sequence in every lane.
__device__ __forceinline__ Seq sequence_of_lane(const Seq& s, int l) {
  return Seq{__builtin_amdgcn_readlane(s.start, l), __builtin_amdgcn_readlane(s.n, l),
             __builtin_amdgcn_readlane(s.kv, l), __builtin_amdgcn_readlane(s.place0, l)};
}

// Where work item `id` lies when a sequence has count(sequence) items: its
// sequence and its number among that sequence's.  Every wave finds it by
// itself, 64 sequences at a time; seq is -1 behind the last item.
struct Found {
  int seq, local;
  Seq s;
};
template <typename Count>
__device__ __forceinline__ Found find_item(const wz_ragged& r, int id, Count count) {
  const int lane = __lane_id();
  int base = 0;
  for (int b0 = 0; b0 < r.batch; b0 += kWave) {
    const bool in = b0 + lane < r.batch;
    const Seq s = in ? sequence(r, b0 + lane) : Seq{0, 0, 0, 0};
    const int c = in ? count(s) : 0, incl = wave_incl_scan_i32(c);
    const int total = __builtin_amdgcn_readlane(incl, kWave - 1);
    if (id - base < total) {
      const int l = __builtin_ctzll(__ballot(incl > id - base));
      const int before = __builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(c, l);
      return Found{b0 + l, id - base - before, sequence_of_lane(s, l)};
    }
    base += total;
  }
  return Found{-1, 0, Seq{}};
}

// The page that `table` entry holds, or -1 where it is none of the cache's.
__device__ __forceinline__ int page_of(const wz_ragged& r, int pages, int b, int entry) {
  const int p = r.table[int64_t(b) * r.table_stride + entry];
  return uint32_t(p) < uint32_t(pages) ? p : -1;
}

// A power of two by its exponent.
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }

struct AppendArgs {
  wz_cache cache;
  wz_ragged batch;
  wz_rotation turn;  // rot_dim 0: none
  const void *k, *v, *q;
  int64_t k_stride, v_stride, q_stride, q_out_stride;
  void* q_out;
  int q_heads;
};
int64_t append_groups(const wz_cache& c, const wz_ragged& r, int q_heads);  // workgroups it launches
hipError_t launch_append(const AppendArgs& a, int in_dtype, hipStream_t s);

struct AttendArgs {
  wz_cache cache;
  wz_ragged batch;
  const void* q;
  void* out;
  float* lse;
  int64_t q_stride, out_stride;
  float scale2;  // the scores' factor times log2(e)
  int q_heads, causal, window;
  int blocks;        // the plan's (attend_plan), for each key/value head
  int workers;       // shared: workgroups that share the blocks' tokens, through the workspace
  int shared;
  int block_rows;    // shared: rows that a block has at most
  float* part;       // shared: [slots][kv_heads][rows of a block][head_dim] unnormalised sums
  float* part_ml;    // shared: [slots][kv_heads][rows of a block][2] maximum (log2) and sum
};
struct AttendPlan {
  int block_rows;    // rows of a block: 16, 32, 64 (token kernel; 64: of 64 elements) or 128 (prompt kernel)
  int groups;        // prompt kernel: of four waves that take a block's tiles in turn
  int blocks;        // upper bound of the batch's blocks, for each key/value head
  int workers;       // shared: workgroups for each key/value head
  int slots;         // of the workspace, for each key/value head
  bool shared;       // several workgroups share a block's tokens
  size_t part_bytes, ml_bytes, bytes;
};
AttendPlan attend_plan(const wz_cache& c, const wz_ragged& r, int q_heads, int window);
hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, hipStream_t s);
hipError_t launch_attend_prompt(const AttendArgs& a, const AttendPlan& p, hipStream_t s);


hipError_t launch_quantize(const void* x, int64_t x_stride, int rows, int cols, int in_dtype, int8_t* q,
                           int64_t q_stride, float* scale, hipStream_t s);
struct MatmulArgs {
  const int8_t *a, *w;
  const float *a_scale, *w_scale, *bias;
  void* out;
  int64_t a_stride, w_stride, out_stride;
  int M, N, K;
};
hipError_t launch_matmul(const MatmulArgs& p, int out_dtype, hipStream_t s);

}  // namespace wz
