/*
 * wavezip_serve.h -- C ABI of the operators that serve condensed tokens on
 * AMD Instinct MI355X (gfx950): one language-model layer's traffic with a
 * paged key/value cache held in 8 bits, and matrix products in 8-bit
 * integers.
 *
 *   wz_cache_append     rotates new keys (and queries) by their positions and
 *                       stores keys and values in the cache;
 *   wz_cache_attention  attention of a ragged batch of queries over the cache;
 *   wz_quantize_rows    rows to 8-bit integers with one scale each;
 *   wz_matmul_int       their product with weights held the same way.
 *
 * The conventions of wavezip.h hold here too: device pointers owned by the
 * caller, nothing allocated or kept by the library, all work enqueued on
 * `stream`, validation before anything is enqueued, bitwise reproducible
 * outputs.  The structs below are read on the host during the call; the
 * arrays they point to are read on the device.
 *
 * The cache.  Memory comes in pages of `page_size` tokens (a power of two,
 * 16 to 128).  A page holds, for each key/value head, its keys as
 * [page_size][head_dim] and its values as [head_dim][page_size] (channel by
 * channel: a product over tokens reads them contiguously) in 8-bit floats
 * (OCP e4m3: 4 significant bits, largest value 448), and one fp32 scale for
 * the keys and one for the values: a stored code c stands for c * scale.
 * Scales are powers of two from 2^-100 to 2^119, so that a page whose scale
 * has to grow is moved to it without a second rounding (but for values that
 * become subnormal).  A sequence's page i, wherever it lies, holds its tokens
 * i * page_size to (i + 1) * page_size - 1.  Nothing in the cache needs
 * initialising: what lies behind a sequence's last token is never used.
 */
#ifndef WAVEZIP_SERVE_H
#define WAVEZIP_SERVE_H

#include <stddef.h>
#include <stdint.h>

#include "wavezip.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The cache of one layer.  Supported: head_dim 64 or 128; page_size 16, 32,
 * 64 or 128; 1 <= kv_heads <= 256; 1 <= pages (pages * kv_heads * page_size *
 * head_dim may pass 2^32).  k and v 16-byte aligned, scales 4-byte.          */
typedef struct {
  void* k;         /* [pages][kv_heads][page_size][head_dim] e4m3             */
  void* v;         /* [pages][kv_heads][head_dim][page_size] e4m3             */
  float* k_scale;  /* [pages][kv_heads]                                       */
  float* v_scale;  /* [pages][kv_heads]                                       */
  int32_t pages, kv_heads, page_size, head_dim;
} wz_cache;

/* A ragged batch: sequence b brings the tokens start[b] .. start[b+1] - 1 of
 * the call's rows and has kv_len[b] tokens in the cache COUNTING those, so
 * its new token i stands at place kv_len[b] - n_b + i of the sequence.
 * Supported: 1 <= batch <= 65536; 0 <= tokens < 2^24; max_tokens and max_kv
 * (bounds that the caller knows for n_b and kv_len[b]) >= 0 and < 2^24;
 * max_kv <= table_stride * page_size.  On the device a start outside
 * [0, tokens], a negative length, an n_b above max_tokens or a kv_len above
 * max_kv is cut to that range, and a page number outside [0, pages) is never
 * followed: its tokens are neither stored nor attended to.  New tokens at a
 * negative place (n_b > kv_len[b]) are not stored, and where attention is
 * causal their rows see nothing.  Distinct sequences may share a page only if
 * none of them brings a token to that page in the call.  A call is refused
 * (WZ_ERR_SHAPE) where its bounds would take more than 2^23 workgroups (pages
 * that receive tokens, or blocks of 16 rows and more, times kv_heads).
 *
 * Attention is planned by the bounds: max_tokens alone decides how many rows
 * work together and by which kernel, for all sequences of the call.  Sequences
 * that bring a token or a few are faster in a call of their own than beside a
 * prompt (a prompt of 1286 rows, 28 heads of 128 over 4, and next tokens of 64
 * sequences of 500 to 8200 tokens: 149 us in one call, 32 and 51 in two; of four
 * of 60 000 to 131 000: 1666, and 34 and 79).                                 */
typedef struct {
  const int32_t* start;   /* [batch + 1], not decreasing                      */
  const int32_t* kv_len;  /* [batch]                                          */
  const int32_t* table;   /* [batch][table_stride] page numbers               */
  int32_t batch, tokens, max_tokens, max_kv, table_stride;
} wz_ragged;

/* Rotation of a head's first rot_dim elements by position.  Frequency j <
 * rot_dim / 2 turns the pair (x_j, x_{j + rot_dim/2}), or (x_{2j}, x_{2j+1})
 * when interleaved, by the angle whose cosine and sine are table[p][j] and
 * table[p][rot_dim/2 + j]:  (a, b) -> (a cos - b sin, b cos + a sin), in fp32
 * without fused multiply-adds.  With axes = 1, p is the token's position;
 * with axes = 2 or 3 (time, row, column of a video token) the frequencies
 * fall into sections of the given lengths and section a uses positions[a].
 * Supported: rot_dim a multiple of 16, 16 to head_dim; axes 1 to 3, sections
 * >= 0 that sum to rot_dim / 2 (axes = 1: sections are not read); max_pos >=
 * 1.  A position outside [0, max_pos) uses the nearest row of the table.      */
typedef struct {
  const float* table;        /* [max_pos][rot_dim] fp32, 16-byte aligned      */
  const int32_t* positions;  /* [axes][tokens]                                */
  int32_t max_pos, rot_dim, axes, interleaved;
  int32_t sections[3];
} wz_rotation;

/* Appends the batch's new tokens to the cache.  k and v are rows of kv_heads
 * heads of head_dim elements of in_dtype (fp32 or bf16), k_stride and
 * v_stride elements apart (multiples of 8, at least kv_heads * head_dim; the
 * pointers 16-byte aligned), so the parts of one fused projection can be
 * passed as they lie.  rotation may be NULL (nothing is rotated); v never is.
 * If q is not NULL its q_heads heads are rotated as well, in all `tokens` rows,
 * and written to q_out (bf16, rows q_out_stride elements apart; q_out must not
 * overlap q).
 *
 * Of every page that receives tokens, keys and values each get the least
 * scale 2^e with |x| <= 448 * 2^e for all its new elements, but no less than
 * the page's scale so far if the sequence already had tokens in it; these are
 * moved to the new scale (code * old / new, rounded to e4m3).  New elements
 * are divided by the scale and rounded to the nearest e4m3, ties to even.
 * Slots of the page that hold none of the sequence's tokens keep their bytes.
 *
 * A NaN or an infinity does not enter a scale.  A token with one in its
 * rotated key or its value, in some head, is stored with a key of NaN there
 * and zeros for those elements of the value: exactly the output rows that
 * attend to it become NaN.
 *
 * One kernel launch; none when the batch has no tokens, or when max_tokens is 0
 * and q NULL.                                                                */
wz_status wz_cache_append(const wz_cache* cache, const wz_ragged* batch,
                          const wz_rotation* rotation, const void* k,
                          int64_t k_stride, const void* v, int64_t v_stride,
                          const void* q, int64_t q_stride, int32_t q_heads,
                          void* q_out, int64_t q_out_stride, int32_t in_dtype,
                          void* stream);

/* What a row attends to.  q_heads is a multiple of kv_heads (at most 64 times
 * it); query head i reads key head i / (q_heads / kv_heads).  causal: a token
 * sees places up to its own; window > 0 (with causal): only the last `window`
 * of them; otherwise every token of its sequence.  scale: finite.            */
typedef struct {
  int32_t q_heads, causal, window;
  float scale;
} wz_attention;

/* Bytes of workspace wz_cache_attention needs (0 if the arguments are invalid
 * or none is needed): partial results of rows whose tokens several
 * workgroups share, at most 128 MiB.  Depends on batch, tokens, max_tokens,
 * max_kv, the head counts and the window alone, not on the arrays' contents. */
size_t wz_attention_workspace_bytes(const wz_cache* cache,
                                    const wz_ragged* batch,
                                    const wz_attention* cfg);

/* Attention over the cache:
 *   out[t][i] = sum_j p_j v_j,  p = softmax_j(scale * q[t][i] . k_j)
 * over the places j that token t sees.  q and out are bf16 rows of q_heads
 * heads, q_stride and out_stride elements apart (multiples of 8; 16-byte
 * aligned).  A row that sees nothing gets zeros.  lse (optional, may be
 * NULL): [tokens][q_heads] fp32, the natural logarithm of the row's sum of
 * exp(scale * q . k) (-inf for a row that sees nothing).  Scores, softmax and
 * sums are fp32; products are bf16 with the cache's values exact in them and
 * the probabilities rounded to bf16 once.  Rows of tokens that no sequence of
 * the batch has are not written.  ws: 256-byte aligned, at least
 * wz_attention_workspace_bytes() bytes; contents on entry are ignored.  One
 * kernel launch, or two when a workspace is needed.                          */
wz_status wz_cache_attention(const wz_cache* cache, const wz_ragged* batch,
                             const wz_attention* cfg, const void* q,
                             int64_t q_stride, void* out, int64_t out_stride,
                             float* lse, void* ws, size_t ws_bytes,
                             void* stream);

/* Rows to 8-bit integers: scale[m] = max(amax, 2^-100) / 127 with amax the
 * row's largest magnitude, q[m][k] = x[m][k] * (127 / max(amax, 2^-100))
 * rounded to the nearest integer, ties to even.  A row with a NaN or an
 * infinity gets the scale NaN and zeros.  x: [rows][cols] of in_dtype, rows
 * x_stride elements apart; q: int8, rows q_stride bytes apart.  Supported:
 * 0 <= rows < 2^24, 16 <= cols <= 65536 a multiple of 16, x_stride a
 * multiple of 8 and q_stride of 16, both >= cols; x and q 16-byte aligned.
 * One kernel launch.                                                         */
wz_status wz_quantize_rows(const void* x, int64_t x_stride, int32_t rows,
                           int32_t cols, int32_t in_dtype, int8_t* q,
                           int64_t q_stride, float* scale, void* stream);

/* The product of quantized rows with quantized weights:
 *   out[m][n] = (sum_k a[m][k] w[n][k]) * a_scale[m] * w_scale[n] + bias[n]
 * with the sum exact in 32-bit integers and the rest in fp32 (the first scale
 * multiplies first), rounded to out_dtype.  a [M][K] and w [N][K] int8, rows
 * a_stride and w_stride bytes apart; out [M][N], rows out_stride elements
 * apart; bias [N] fp32 or NULL.  Supported: 0 <= M < 2^24; 1 <= N < 2^24; M * N
 * <= 2^38; 16 <= K <= 65536 (a sum is then at most 2^30), a multiple of 16; a_stride,
 * w_stride multiples of 16, K to 2^22; out_stride >= N; a and w 16-byte
 * aligned, out aligned to its element.  One kernel launch, or two (the rows of
 * whole rounds of large tiles, and those behind them).                       */
wz_status wz_matmul_int(const int8_t* a, int64_t a_stride,
                        const float* a_scale, const int8_t* w,
                        int64_t w_stride, const float* w_scale,
                        const float* bias, int32_t M, int32_t N, int32_t K,
                        void* out, int64_t out_stride, int32_t out_dtype,
                        void* stream);

#ifdef __cplusplus
}
#endif

#endif /* WAVEZIP_SERVE_H */
