// Internal launch interface of the 8-bit cache's calls and the rotation,
// between the C ABI (abi_q8.cpp) and the HIP kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "internal.h"
#include "mbe_q8.h"

namespace mbe {

// ------------------------------------------------------- quantised pages
struct KvQ8Params {
  uint8_t *k_pages;          // [num_pages][Hkv][16][D]
  uint8_t *v_pages;          // [num_pages][Hkv][D][16]
  float *k_scales, *v_scales;        // [num_pages][Hkv]
  int32_t num_pages, num_kv_heads;
  const int32_t *page_table;         // [batch][max_pages]
  int32_t max_pages;
  const int32_t *start_pos, *lens;
  const int32_t *kv_lens;            // write: tokens held before the call, or null (= start_pos)
  int32_t batch, max_len, total_tokens;
  const uint16_t *k_new, *v_new;     // write: bf16 [total_tokens][heads][D]
  uint16_t *k_out, *v_out;           // read:  bf16 [total_tokens][heads][D]
  const uint8_t *block_flags;        // write: [batch][flag_stride] or null
  int32_t block_size, flag_stride;
};
hipError_t launch_kv_write_q8(const KvQ8Params &p, int head_dim, int format, hipStream_t stream);
hipError_t launch_kv_read_q8(const KvQ8Params &p, int head_dim, int format, hipStream_t stream);

// ---------------------------------------------------------------- rotation
struct RotaryParams {
  const uint16_t *q, *k;             // bf16 rows, `*_stride` values apart
  uint16_t *q_out, *k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
  int32_t num_q_heads, num_kv_heads;
  const int32_t *start_pos, *lens;
  int32_t batch, max_len, total_rows;
  const uint64_t *turns;             // [rot_dim / 2], units of 2^-64 turns per position
  int32_t rot_dim, interleaved, inverse;
  float scale;
};
hipError_t launch_rotary(const RotaryParams &p, int head_dim, hipStream_t stream);

// --------------------------------------------------------------- attention
struct AttnQ8Params {
  const uint16_t *q;                 // bf16 [total_q][Hq][D]
  const uint8_t *k_pages, *v_pages;
  const float *k_scales, *v_scales;
  const int32_t *page_table;         // [batch][max_pages]
  const int32_t *prefix_lens, *window_lens;
  uint16_t *out;                     // bf16 [total_q][Hq][D]
  int32_t *notes;                    // [wgs][8]                   (split only; see attn_q8.hip)
  float *part_o;                     // fp32 [2 * wgs][rows][D]
  float *part_ml;                    // fp32 [2 * wgs][rows][2]
  int32_t batch, num_q_heads, num_kv_heads, group, num_pages, max_pages;
  int32_t block_size, total_q, max_prefix, max_window, causal;
  float scale_log2;                  // softmax scale * log2(e)
  const uint8_t *block_flags;        // [batch][flag_stride] or null
  int32_t flag_stride;
  const int32_t *gate;               // device int32 or null: nothing is done when *gate == 0
  int32_t wgs;                       // workgroups
  int32_t min_tiles;                 // fewest 64-key tiles of a workgroup's share
  int32_t start_tiles;               // tiles' time that beginning a unit takes
  int32_t memory_tiles;              // tiles the memory delivers in a workgroup's time for one
  int32_t join_tiles;                // tiles' time that joining parts takes
  int32_t qtiles;                    // row tiles of the widest window
  int32_t split;                     // 0: a workgroup takes one whole unit
};

// Launch shape of the attention, from host-known bounds.
struct AttnQ8Plan {
  int32_t rows;       // packed query rows of a unit
  int32_t qtiles, wgs, min_tiles, start_tiles, memory_tiles, join_tiles, split;
  size_t part_o_off, part_ml_off, bytes;
};
hipError_t launch_attn_q8(const AttnQ8Params &p, const AttnQ8Plan &plan, int head_dim, int format, hipStream_t stream);

}  // namespace mbe
