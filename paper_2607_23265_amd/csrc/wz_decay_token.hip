// Linear attention with a decay for each head, token after token
// (wz_decay_attention).
#include "wz_decay.h"

namespace wz {
namespace {

// S <- l S + k v^T, out = scale q S, as they are written, in fp32.  A wave has 32
// columns of a sequence's and head's state, four a lane, and a lane D / 8 of
// their rows: what a row's 128 bytes of state need is read and written whole, and a
// token's output is a sum over eight lanes.  Few waves of many loads each: a state is
// read and written once, and that bounds it.  Measured with states that come from memory
// (28 heads of 128 elements): the next tokens of 64 sequences, 235 MB, in 48.0 to 48.5 us,
// 4.9 TB/s (a large copy: 5.1 to 5.2; with the states in the last-level cache 37 us); of one
// sequence 4.4 to 5.5 us, where an empty launch takes 3.6.  Heads of 64 elements: 16.3 and 3.9.
template <int D>
__global__ __launch_bounds__(kWave) void k_decay_token(DecayArgs p) {
  constexpr int kRows = D / 8;  // of a lane
  const int lane = __lane_id(), col = lane & 7, part = lane >> 3;
  const int slice = blockIdx.x % (D / 32), h = blockIdx.x / (D / 32) % p.states.heads;
  const int b = blockIdx.x / (D / 32) / p.states.heads;
  const Seq s = sequence(p.batch, b);
  if (s.n <= 0) return;
  const int kh = h / p.group;
  const int slot = p.slot[b];
  const bool kept = uint32_t(slot) < uint32_t(p.states.slots);
  float* const state = p.states.state + (int64_t(kept ? slot : 0) * p.states.heads + h) * (D * D) +
                       part * kRows * D + slice * 32 + 4 * col;
  f32x4 S[kRows] = {};
  if (kept && s.place0 > 0) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) S[i] = *reinterpret_cast<const f32x4*>(state + i * D);
  }
  // The factor in two parts: rounded to one, it would be off the same way for
  // every token of a long answer (by 2^-25 each).
  const double factor = exp2(double(log2_decay(p, h)));
  const float l = float(factor), l2 = float(factor - l);
  const uint16_t* q = static_cast<const uint16_t*>(p.q) + s.start * p.q_stride + h * D + part * kRows;
  const uint16_t* k = static_cast<const uint16_t*>(p.k) + s.start * p.k_stride + kh * D + part * kRows;
  const uint16_t* v = static_cast<const uint16_t*>(p.v) + s.start * p.v_stride + kh * D + slice * 32 + 4 * col;
  uint16_t* out = static_cast<uint16_t*>(p.out) + s.start * p.out_stride + h * D + slice * 32 + 4 * col + (part & 3);
  for (int t = 0; t < s.n; ++t) {
    u32x4 qv[kRows / 8], kv[kRows / 8];
#pragma unroll
    for (int i = 0; i < kRows / 8; ++i) {
      qv[i] = *reinterpret_cast<const u32x4*>(q + 8 * i);
      kv[i] = *reinterpret_cast<const u32x4*>(k + 8 * i);
    }
    const u32x2 vv = *reinterpret_cast<const u32x2*>(v);
    const float ve[4] = {bf16_lo(vv[0]), bf16_hi(vv[0]), bf16_lo(vv[1]), bf16_hi(vv[1])};
    float o[4] = {};
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const uint32_t qw = qv[i / 8][i % 8 / 2], kw = kv[i / 8][i % 8 / 2];
      const float qe = i % 2 ? bf16_hi(qw) : bf16_lo(qw), ke = i % 2 ? bf16_hi(kw) : bf16_lo(kw);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        S[i][e] = fmaf(S[i][e], l, fmaf(S[i][e], l2, ke * ve[e]));
        o[e] = fmaf(qe, S[i][e], o[e]);
      }
    }
    const float y = lane_transpose_sum(o) * p.scale;  // of column `part & 3`
    if (part < 4) *out = __builtin_bit_cast(uint16_t, __bf16(y));
    q += p.q_stride, k += p.k_stride, v += p.v_stride, out += p.out_stride;
  }
  if (kept) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) *reinterpret_cast<f32x4*>(state + i * D) = S[i];
  }
}

}  // namespace

hipError_t launch_decay_token(const DecayArgs& p, hipStream_t s) {
  const uint32_t grid = uint32_t(p.batch.batch) * p.states.heads * (p.states.head_dim / 32);
  if (p.states.head_dim == 128) hipLaunchKernelGGL((k_decay_token<128>), dim3(grid), dim3(kWave), 0, s, p);
  else hipLaunchKernelGGL((k_decay_token<64>), dim3(grid), dim3(kWave), 0, s, p);
  return hipGetLastError();
}

}  // namespace wz
