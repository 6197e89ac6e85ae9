/*
 * mbe_q8.h -- C ABI of libmbe: the 8-bit KV cache of a decoding loop and the
 * rotation of its queries and keys, for AMD MI355X (gfx950).
 *
 * From a layer's projected q, k, v to its attention output:
 *   mbe_rotary               q and k rotated by their absolute positions
 *   mbe_kv_write_q8          k and v quantised into 8-bit pages
 *   mbe_window_attention_q8  window queries over the 8-bit cache
 *   mbe_kv_read_q8           ranges of the cache read back as bf16
 *
 * The conventions of mbe.h hold for every call: device memory owned by the
 * caller, asynchronous on `stream`, kernels on the current HIP device,
 * arguments checked on the host before anything is launched, errors through
 * mbe_status and mbe_last_error().  No call allocates or synchronises, except
 * under MBE_DEBUG_CHECK=1, where the calls that take a page table copy it and
 * the lengths to the host, check them, and return MBE_ERR_BAD_VALUE on a
 * violation (not while the stream is being captured).
 */
#ifndef MBE_Q8_H_
#define MBE_Q8_H_

#include "mbe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* 8-bit types of a pool (OCP): e4m3 (finite up to 448, no infinities) and
 * e5m2 (finite up to 57344). */
typedef enum { MBE_Q8_E4M3 = 0, MBE_Q8_E5M2 = 1 } mbe_q8_format;

/* Paged 8-bit KV cache for one layer.  Pages hold 16 tokens.
 *   k_pages:  [num_pages][num_kv_heads][16][head_dim]   one byte a value
 *   v_pages:  [num_pages][num_kv_heads][head_dim][16]   (token-minor)
 *   k_scales, v_scales: float [num_pages][num_kv_heads]
 * A value of page p and head h is its 8-bit value times the scale [p][h].
 * Token t of sequence b is slot t % 16 of page page_table[b][t / 16].
 * mbe_kv_write_q8 stores scales that are powers of two; the other calls take
 * any positive finite scale (mbe_window_attention_q8 takes those of V as at
 * least 2^-100 and at most 2^100).
 * The slots that no sequence covers, and the scales of pages without a
 * covered slot, may hold anything, NaN included. */
typedef struct {
  void *k_pages;
  void *v_pages;
  float *k_scales;
  float *v_scales;
  int32_t num_pages;
  int32_t page_size;     /* must be 16            */
  int32_t num_kv_heads;  /* Hkv >= 1              */
  int32_t head_dim;      /* D: 64 or 128          */
  int32_t format;        /* mbe_q8_format         */
} mbe_paged_kv_q8;

/* Quantising write.  Token t < lens[b] of sequence b (rows of sequence b start
 * at sum_{b' < b} lens[b']) is written at position start_pos[b] + t for every
 * KV head.  k_new/v_new: bf16 [total_tokens][num_kv_heads][head_dim].
 *
 * On every page with a written slot, for K and for V and each head:
 *   new slots   written by this call
 *   kept slots  the others at positions below max(start_pos[b], kv_lens[b])
 *   amax        largest finite magnitude of the new values
 *   s           smallest power of two, in [2^-100, 2^120], with
 *               amax / s <= the type's largest finite value
 *   scale       s, or max(s, old scale) where a slot is kept
 *   new value   x / scale (in fp32: exact for powers of two), rounded to the
 *               nearest 8-bit value, ties to even; +-inf becomes the largest
 *               finite value, NaN stays NaN
 *   kept value  old value * (old scale / scale), rounded likewise
 * The remaining slots keep their bytes.  kv_lens (device int32 [batch], NULL =
 * start_pos): tokens the sequence holds before the call.  An append passes
 * NULL; a call that writes over tokens in the middle of a sequence must pass
 * the sequence's length, or the tokens behind the written range on its last
 * page lose their scale.
 * max_len bounds every lens[b].  block_flags, block_size: as for mbe_kv_write
 * (a token of an unflagged block is not written; it is kept when its position
 * is below max(start_pos[b], kv_lens[b])).
 * A page must not be written for two sequences in one call.
 * A token whose table slot or page id is out of range is not written. */
mbe_status mbe_kv_write_q8(const mbe_paged_kv_q8 *paged_kv, const int32_t *page_table, int32_t max_pages_per_seq,
                           const int32_t *start_pos, const int32_t *lens, const int32_t *kv_lens, int32_t batch,
                           int32_t max_len, int32_t total_tokens, const void *k_new, const void *v_new,
                           const uint8_t *block_flags, int32_t block_size, void *stream);

/* Read-back: the tokens at positions start_pos[b] .. start_pos[b] + lens[b] - 1
 * of every sequence as bf16 [total_tokens][num_kv_heads][head_dim], rows as in
 * mbe_kv_write_q8.  Each value is the 8-bit value times its scale, in fp32,
 * rounded to bf16 (exact for the scales mbe_kv_write_q8 stores, down to bf16's
 * smallest normal value).  Tokens whose table slot or page id is out of range read as
 * zeros; rows behind the last sequence are left as they were. */
mbe_status mbe_kv_read_q8(const mbe_paged_kv_q8 *paged_kv, const int32_t *page_table, int32_t max_pages_per_seq,
                          const int32_t *start_pos, const int32_t *lens, int32_t batch, int32_t max_len,
                          int32_t total_tokens, void *k_out, void *v_out, void *stream);

/* mbe_window_attention over an 8-bit cache.  q, out, page_table, the lengths,
 * block_size and opts are those of mbe_window_attention, with two options
 * read differently:
 *   kv_split_tokens  the fewest keys that a workgroup takes of a sequence
 *                    before the sequence is split further; 0 lets the library
 *                    choose (and take smaller tiles of rows where there is
 *                    little to do); otherwise a positive multiple of 64
 *   host_prefix_lens, host_window_lens   not read: the work is dealt out on the
 *                    device, from the device lengths
 * q and the probabilities take part in full bf16 precision; the cache's values
 * are never rounded again; accumulation is fp32.  Deterministic: the same
 * inputs and bounds give bitwise the same outputs.
 * A row of q that holds an infinity or a NaN gives NaN, in that row alone.
 * V values that a row's scope hides within a sequence's own tokens (block-causal
 * windows) must be finite, as must the scales of all covered pages. */
mbe_status mbe_window_attention_q8(const void *q, const mbe_paged_kv_q8 *paged_kv, const int32_t *page_table,
                                   const int32_t *prefix_lens, const int32_t *window_lens, int32_t block_size,
                                   void *out, const mbe_attn_opts *opts);

/* Workspace bytes mbe_window_attention_q8 needs for these shapes and options
 * (bounds only; 0 = none).  (size_t)-1 if the arguments are invalid. */
size_t mbe_window_attention_q8_workspace_size(const mbe_paged_kv_q8 *paged_kv, const mbe_attn_opts *opts);

/* Pairing of the rotated dims: HALF pairs dim i with dim i + rot_dim / 2,
 * INTERLEAVED pairs dim 2i with dim 2i + 1, for i < rot_dim / 2. */
typedef enum { MBE_ROTARY_HALF = 0, MBE_ROTARY_INTERLEAVED = 1 } mbe_rotary_layout;

/* Rotary positions.  Row t < lens[b] of sequence b (rows of sequence b start
 * at sum_{b' < b} lens[b']) is at position n = start_pos[b] + t.  For every
 * head of q and of k, pair i (x, y) of the row becomes
 *   scale * (x cos a - y sin a),  scale * (y cos a + x sin a),
 *   a = 2 pi * frac(n * turns[i] / 2^64)
 * and the dims from rot_dim on are copied.  turns: device int64 [rot_dim / 2],
 * the turns per position of each pair in units of 2^-64 (a frequency of f
 * radians per position is round(f / (2 pi) * 2^64), modulo 2^64): the phase is
 * exact at any position.  Frequencies scaled for long contexts are a matter of
 * this table, a factor on the attention's logits one of `scale`.
 * inverse != 0 rotates by -a: the transpose of the same map, which is its
 * gradient (and for scale 1 undoes it).
 * q, k: bf16 rows of num_q_heads (num_kv_heads) * head_dim values; consecutive
 * rows are q_stride (k_stride) values apart, so both may lie in one packed
 * projection; outputs likewise.  An output may be its own input (same pointer
 * and stride); otherwise it must not overlap an input.  k may be NULL with
 * num_kv_heads = 0, and q with num_q_heads = 0.  Arithmetic is fp32, rounded
 * once.  Rows behind the last sequence are left as they were.
 * rot_dim: a multiple of 16, at most head_dim.  Pointers must be 16-byte
 * aligned and strides multiples of 8. */
mbe_status mbe_rotary(const void *q, void *q_out, int32_t num_q_heads, int64_t q_stride, int64_t q_out_stride,
                      const void *k, void *k_out, int32_t num_kv_heads, int64_t k_stride, int64_t k_out_stride,
                      int32_t head_dim, const int32_t *start_pos, const int32_t *lens, int32_t batch, int32_t max_len,
                      int32_t total_rows, const int64_t *turns, int32_t rot_dim, int32_t layout, float scale,
                      int32_t inverse, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* MBE_Q8_H_ */
