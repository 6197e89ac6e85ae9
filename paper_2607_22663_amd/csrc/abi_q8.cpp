// C ABI of the 8-bit cache's calls and the rotation: argument checks, launch
// planning and dispatch.  Every check runs before the first HIP call, so the
// validation paths work on a machine without a GPU.
#include "mbe_q8.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <new>
#include <vector>

#include "q8.h"

namespace {

using mbe::report;

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
constexpr int64_t kMaxGrid = (1LL << 24) - 1;      // workgroups of 256 threads in one dimension

mbe_status hip_error(hipError_t e, const char *where) {
  return report(MBE_ERR_HIP, "%s: %s", where, hipGetErrorString(e));
}

bool misaligned(std::initializer_list<const void *> ptrs, uintptr_t align) {
  uintptr_t bits = 0;
  for (const void *q : ptrs) bits |= reinterpret_cast<uintptr_t>(q);
  return bits % align != 0;
}

mbe_status check_pool(const mbe_paged_kv_q8 *kv) {
  if (!kv) return report(MBE_ERR_NULL_ARG, "paged_kv is NULL");
  if (kv->page_size != mbe::kPageSize)
    return report(MBE_ERR_UNSUPPORTED, "page_size %d: only 16-token pages are supported", kv->page_size);
  if (kv->head_dim != 64 && kv->head_dim != 128)
    return report(MBE_ERR_UNSUPPORTED, "head_dim %d: supported are 64 and 128", kv->head_dim);
  if (kv->format != MBE_Q8_E4M3 && kv->format != MBE_Q8_E5M2)
    return report(MBE_ERR_UNSUPPORTED, "format %d", kv->format);
  if (kv->num_kv_heads < 1 || kv->num_kv_heads > 65535)
    return report(MBE_ERR_BAD_SHAPE, "num_kv_heads %d outside [1, 65535]", kv->num_kv_heads);
  if (kv->num_pages < 0) return report(MBE_ERR_BAD_SHAPE, "num_pages %d < 0", kv->num_pages);
  return MBE_OK;
}

mbe_status check_pool_pointers(const mbe_paged_kv_q8 *kv) {
  if (!kv->k_pages || !kv->v_pages || !kv->k_scales || !kv->v_scales)
    return report(MBE_ERR_NULL_ARG, "k_pages, v_pages, k_scales and v_scales must be non-NULL");
  if (misaligned({kv->k_pages, kv->v_pages}, 16)) return report(MBE_ERR_BAD_SHAPE, "pools must be 16-byte aligned");
  if (misaligned({kv->k_scales, kv->v_scales}, 4)) return report(MBE_ERR_BAD_SHAPE, "scales must be 4-byte aligned");
  return MBE_OK;
}

// ---------------------------------------------------------- MBE_DEBUG_CHECK
bool debug_checks() {
  const char *v = std::getenv("MBE_DEBUG_CHECK");
  return v && v[0] == '1';
}

// The ranges [start, start + len) of every sequence against the table, the pool
// and the rows; `what` names the lengths.
mbe_status debug_check_ranges(const mbe_paged_kv_q8 *kv, const int32_t *page_table, int32_t max_pages,
                              const int32_t *start, const int32_t *lens, int32_t batch, int32_t max_start,
                              int32_t max_len, int32_t multiple_of, int32_t total, bool whole, hipStream_t stream) try {
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  hipError_t e = hipStreamIsCapturing(stream, &cs);
  if (e != hipSuccess) return hip_error(e, "MBE_DEBUG_CHECK capture query");
  if (cs != hipStreamCaptureStatusNone) return MBE_OK;
  std::vector<int32_t> S(batch), L(batch), T(static_cast<size_t>(batch) * max_pages);
  e = hipMemcpyAsync(S.data(), start, batch * sizeof(int32_t), hipMemcpyDeviceToHost, stream);
  if (e == hipSuccess) e = hipMemcpyAsync(L.data(), lens, batch * sizeof(int32_t), hipMemcpyDeviceToHost, stream);
  if (e == hipSuccess && !T.empty())
    e = hipMemcpyAsync(T.data(), page_table, T.size() * sizeof(int32_t), hipMemcpyDeviceToHost, stream);
  const hipError_t done = hipStreamSynchronize(stream);
  if (e != hipSuccess || done != hipSuccess) return hip_error(e != hipSuccess ? e : done, "MBE_DEBUG_CHECK copy");
  int64_t rows = 0;
  for (int b = 0; b < batch; ++b) {
    if (S[b] < 0 || S[b] > max_start)
      return report(MBE_ERR_BAD_VALUE, "sequence %d starts at %d, outside [0, %d]", b, S[b], max_start);
    if (L[b] < 0 || L[b] > max_len || L[b] % multiple_of != 0)
      return report(MBE_ERR_BAD_VALUE, "length %d of sequence %d is not a multiple of %d in [0, %d]", L[b], b,
                    multiple_of, max_len);
    rows += L[b];
    if (L[b] == 0) continue;
    const int64_t last = (static_cast<int64_t>(S[b]) + L[b] - 1) / mbe::kPageSize;
    if (last >= max_pages)
      return report(MBE_ERR_BAD_VALUE, "sequence %d needs %lld pages, its table row has %d", b,
                    static_cast<long long>(last + 1), max_pages);
    for (int64_t j = whole ? 0 : S[b] / mbe::kPageSize; j <= last; ++j) {
      const int32_t pg = T[static_cast<size_t>(b) * max_pages + j];
      if (pg < 0 || pg >= kv->num_pages)
        return report(MBE_ERR_BAD_VALUE, "page_table[%d][%lld] = %d outside [0, %d)", b, static_cast<long long>(j), pg,
                      kv->num_pages);
    }
  }
  if (rows != total)
    return report(MBE_ERR_BAD_VALUE, "the lengths add up to %lld, the rows to %d", static_cast<long long>(rows), total);
  return MBE_OK;
} catch (const std::bad_alloc &) {
  return report(MBE_ERR_BAD_VALUE, "MBE_DEBUG_CHECK: no host memory for a copy of the page table");
}

// ------------------------------------------------------- ranges of a pool
mbe_status check_ranges(const mbe_paged_kv_q8 *kv, int32_t max_pages, int32_t batch, int32_t max_len,
                        int32_t total_tokens) {
  const mbe_status st = check_pool(kv);
  if (st != MBE_OK) return st;
  if (batch < 0 || batch > 65535) return report(MBE_ERR_BAD_SHAPE, "batch %d outside [0, 65535]", batch);
  if (max_len < 0 || total_tokens < 0 || max_pages < 0)
    return report(MBE_ERR_BAD_SHAPE, "negative max_len/total_tokens/max_pages_per_seq");
  if ((static_cast<int64_t>(max_len) / mbe::kPageSize + 2) * 2 * kv->num_kv_heads / 4 >= kMaxGrid)
    return report(MBE_ERR_BAD_SHAPE, "max_len %d x %d heads is too large for one call", max_len, kv->num_kv_heads);
  return MBE_OK;
}

mbe::KvQ8Params range_params(const mbe_paged_kv_q8 *kv, const int32_t *page_table, int32_t max_pages,
                             const int32_t *start_pos, const int32_t *lens, int32_t batch, int32_t max_len,
                             int32_t total_tokens) {
  mbe::KvQ8Params p{};
  p.k_pages = static_cast<uint8_t *>(kv->k_pages);
  p.v_pages = static_cast<uint8_t *>(kv->v_pages);
  p.k_scales = kv->k_scales;
  p.v_scales = kv->v_scales;
  p.num_pages = kv->num_pages;
  p.num_kv_heads = kv->num_kv_heads;
  p.page_table = page_table;
  p.max_pages = max_pages;
  p.start_pos = start_pos;
  p.lens = lens;
  p.batch = batch;
  p.max_len = max_len;
  p.total_tokens = total_tokens;
  p.block_size = 1;
  return p;
}

// --------------------------------------------------------------- attention
// Shares of the work: one workgroup on each of the 256 CUs.  (Two of the streaming
// kernel, main kernel: one token of 32 sequences of 1000 to 8192 37 against 33 us,
// of 32 x 65536 381 against 355.)
constexpr int64_t kWgs = 256;
// Smallest share where units are cut.  1 x 8192 / 8 x 2048 keys, us, with shares of
// at least 2 / 4 / 8 tiles: one token 13.4 12.9 12.9 / 13.2 13.1 12.7, windows of 32
// 33 29 28 / 28 28 29, of 64 37 37 37 / 36 36 38; 1 x 1024, windows of 64 22 23 29.
constexpr int32_t kMinTiles = 4;
// Tiles' time that beginning a unit takes a workgroup (q, the first pages, the
// result).  Main kernel, us, at 0 / 4 / 8 / 12: one token of 32 sequences of 1000
// to 8192 39 / 37 / 37 / 37, blocks behind 8 x 16384 65 / 61 / 59 / 57, 12 ragged
// windows behind 1000 to 12000 132 / 123 / 120 / 121, windows of 128 behind 64 x
// 4096 to 32768 1204 / 1174 / 1154 / 1146.
constexpr int32_t kStartTiles = 8;
// Units of 32 rows for any window while there is little to do, in tiles (and
// starts) of such units: they begin in half the time, and spread wider.  us with
// units of 32 rows / the best of 64 to 256, by that number: windows of 32, 8 x 64
// (1300) 7.5 / 11, 8 x 512 (2200) 11 / 21, 8 x 2048 (5200) 23 / 28, 32 x 512 (8700)
// 19 / 23, 8 x 8192 (17500) 51 / 40; of 16, 32 x 2048 (10500) 30 / 37; of 64, 8 x
// 2048 (10500) 30 / 34, 32 x 64 (10200) 19 / 16, 8 x 8192 (35000) 85 / 59; of 256,
// 1 x 2048 (5600) 21 / 26, 1 x 8192 (17900) 50 / 40.
constexpr int64_t kLittleWork = 11000;
// By units of 32, of 64 and 128, of 256 rows.  A workgroup alone takes 0.29, 0.88,
// 1.46 us a tile (D = 128), the memory 2.8 ns; parts cost about 5 us to join.
constexpr int32_t kMemoryTiles[3] = {100, 300, 500};
constexpr int32_t kJoinTiles[3] = {8, 4, 2};
// Longest units that are not cut at all, without a look at the lengths: one kernel.
constexpr int32_t kWholeTiles[3] = {16, 8, 8};

mbe_status plan_attention(const mbe_paged_kv_q8 *kv, const mbe_attn_opts *o, int32_t block_size, mbe::AttnQ8Plan *pl) {
  const mbe_status st = check_pool(kv);
  if (st != MBE_OK) return st;
  if (!o) return report(MBE_ERR_NULL_ARG, "opts is NULL");
  if (o->batch < 0) return report(MBE_ERR_BAD_SHAPE, "batch %d < 0", o->batch);
  if (o->num_q_heads < 1 || o->num_q_heads % kv->num_kv_heads != 0)
    return report(MBE_ERR_BAD_SHAPE, "num_q_heads %d is not a positive multiple of num_kv_heads %d", o->num_q_heads,
                  kv->num_kv_heads);
  if (block_size < 1) return report(MBE_ERR_BAD_SHAPE, "block_size %d < 1", block_size);
  if (o->total_q < 0 || o->max_prefix_len < 0 || o->max_window_len < 0 || o->max_pages_per_seq < 0)
    return report(MBE_ERR_BAD_SHAPE, "negative total_q/max_prefix_len/max_window_len/max_pages_per_seq");
  if (o->max_window_len % block_size != 0)
    return report(MBE_ERR_BAD_SHAPE, "max_window_len %d is not a multiple of block_size %d", o->max_window_len,
                  block_size);
  if (o->mask_mode != MBE_MASK_WINDOW_BIDIR && o->mask_mode != MBE_MASK_BLOCK_CAUSAL)
    return report(MBE_ERR_UNSUPPORTED, "mask_mode %d", o->mask_mode);
  if (!std::isfinite(o->softmax_scale)) return report(MBE_ERR_BAD_VALUE, "softmax_scale is not finite");
  if (o->kv_split_tokens < 0 || o->kv_split_tokens % mbe::kKeyTile != 0)
    return report(MBE_ERR_BAD_SHAPE, "kv_split_tokens %d is not 0 or a positive multiple of 64", o->kv_split_tokens);
  const int64_t max_kv = static_cast<int64_t>(o->max_prefix_len) + o->max_window_len;
  const int64_t group = o->num_q_heads / kv->num_kv_heads;
  if (max_kv > (1LL << 30) || group * o->max_window_len > (1LL << 30))
    return report(MBE_ERR_BAD_SHAPE, "sequence bound too large");
  if (o->batch > 0 && max_kv > 0 && (o->max_pages_per_seq < 1 || kv->num_pages < 1))
    return report(MBE_ERR_BAD_SHAPE, "empty page pool or table");

  *pl = mbe::AttnQ8Plan{};
  const int64_t seq_rows = group * o->max_window_len;
  const int64_t tiles = (max_kv + mbe::kKeyTile - 1) / mbe::kKeyTile;
  constexpr int64_t kCounted = 1LL << 32;       // (more than any call may have; times heads, within 64 bits)
  // units of `rows` rows within the bounds: no more than the rows fill
  auto units_of = [&](int64_t rows) {
    const int64_t each = (seq_rows + rows - 1) / rows;
    const int64_t all = std::min<int64_t>(o->batch * each, o->total_q * group / rows + o->batch);
    return std::max<int64_t>(1, std::min(all, kCounted) * kv->num_kv_heads);
  };
  const bool little = o->kv_split_tokens == 0 && units_of(32) <= kLittleWork / (tiles + kStartTiles);
  pl->rows = seq_rows <= 32 || little ? 32 : seq_rows <= 64 ? 64 : seq_rows <= 128 ? 128 : 256;
  const int form = pl->rows == 32 ? 0 : pl->rows <= 128 ? 1 : 2;
  const int64_t qtiles = (seq_rows + pl->rows - 1) / pl->rows;
  const int64_t units = units_of(pl->rows);
  const int64_t grid = std::max<int64_t>(1, std::min(o->batch * qtiles, kCounted) * kv->num_kv_heads);
  pl->qtiles = static_cast<int32_t>(std::max<int64_t>(1, qtiles));
  pl->min_tiles = o->kv_split_tokens > 0 ? o->kv_split_tokens / mbe::kKeyTile : kMinTiles;
  // (the kernels count the tiles of all units in 32 bits, whatever the lengths within the bounds)
  pl->start_tiles = kStartTiles;
  pl->memory_tiles = kMemoryTiles[form];
  pl->join_tiles = o->kv_split_tokens > 0 ? 0 : kJoinTiles[form];
  pl->split = tiles > (o->kv_split_tokens > 0 ? pl->min_tiles : kWholeTiles[form]) && grid <= kMaxGrid &&
              grid * (tiles + kStartTiles) < (1LL << 31);
  if (!pl->split && grid > kMaxGrid) return report(MBE_ERR_BAD_SHAPE, "too many sequences, heads and rows for one call");
  if (!pl->split) {
    pl->wgs = static_cast<int32_t>(grid);
    return MBE_OK;
  }
  const int64_t most = units * ((tiles + pl->min_tiles - 1) / pl->min_tiles);
  pl->wgs = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(kWgs, most)));
  const size_t part_rows = 2 * static_cast<size_t>(pl->wgs) * pl->rows;
  pl->part_o_off = align_up(static_cast<size_t>(pl->wgs) * 8 * sizeof(int32_t));
  pl->part_ml_off = pl->part_o_off + align_up(part_rows * kv->head_dim * sizeof(float));
  pl->bytes = pl->part_ml_off + align_up(part_rows * 2 * sizeof(float));
  return MBE_OK;
}

}  // namespace

extern "C" {

mbe_status mbe_kv_write_q8(const mbe_paged_kv_q8 *paged_kv, const int32_t *page_table, int32_t max_pages_per_seq,
                           const int32_t *start_pos, const int32_t *lens, const int32_t *kv_lens, int32_t batch,
                           int32_t max_len, int32_t total_tokens, const void *k_new, const void *v_new,
                           const uint8_t *block_flags, int32_t block_size, void *stream) {
  mbe_status st = check_ranges(paged_kv, max_pages_per_seq, batch, max_len, total_tokens);
  if (st != MBE_OK) return st;
  if (block_flags && block_size < 1) return report(MBE_ERR_BAD_SHAPE, "block_size %d < 1 with block flags", block_size);
  if (batch == 0 || max_len == 0 || total_tokens == 0) return MBE_OK;
  if (paged_kv->num_pages < 1 || max_pages_per_seq < 1) return report(MBE_ERR_BAD_SHAPE, "empty page pool or table");
  st = check_pool_pointers(paged_kv);
  if (st != MBE_OK) return st;
  if (!page_table || !start_pos || !lens || !k_new || !v_new)
    return report(MBE_ERR_NULL_ARG, "page_table, start_pos, lens, k_new and v_new must be non-NULL");
  if (misaligned({k_new, v_new}, 16)) return report(MBE_ERR_BAD_SHAPE, "k_new and v_new must be 16-byte aligned");
  const hipStream_t hs = static_cast<hipStream_t>(stream);
  if (debug_checks()) {
    st = debug_check_ranges(paged_kv, page_table, max_pages_per_seq, start_pos, lens, batch, INT32_MAX, max_len, 1,
                            total_tokens, false, hs);
    if (st != MBE_OK) return st;
  }
  mbe::KvQ8Params p = range_params(paged_kv, page_table, max_pages_per_seq, start_pos, lens, batch, max_len, total_tokens);
  p.kv_lens = kv_lens;
  p.k_new = static_cast<const uint16_t *>(k_new);
  p.v_new = static_cast<const uint16_t *>(v_new);
  p.block_flags = block_flags;
  if (block_flags) {
    p.block_size = block_size;
    p.flag_stride = static_cast<int32_t>((static_cast<int64_t>(max_len) + block_size - 1) / block_size);
  }
  const hipError_t e = mbe::launch_kv_write_q8(p, paged_kv->head_dim, paged_kv->format, hs);
  return e == hipSuccess ? MBE_OK : hip_error(e, "quantising write launch");
}

mbe_status mbe_kv_read_q8(const mbe_paged_kv_q8 *paged_kv, const int32_t *page_table, int32_t max_pages_per_seq,
                          const int32_t *start_pos, const int32_t *lens, int32_t batch, int32_t max_len,
                          int32_t total_tokens, void *k_out, void *v_out, void *stream) {
  mbe_status st = check_ranges(paged_kv, max_pages_per_seq, batch, max_len, total_tokens);
  if (st != MBE_OK) return st;
  if (batch == 0 || max_len == 0 || total_tokens == 0) return MBE_OK;
  if (paged_kv->num_pages < 1 || max_pages_per_seq < 1) return report(MBE_ERR_BAD_SHAPE, "empty page pool or table");
  st = check_pool_pointers(paged_kv);
  if (st != MBE_OK) return st;
  if (!page_table || !start_pos || !lens || !k_out || !v_out)
    return report(MBE_ERR_NULL_ARG, "page_table, start_pos, lens, k_out and v_out must be non-NULL");
  if (misaligned({k_out, v_out}, 16)) return report(MBE_ERR_BAD_SHAPE, "k_out and v_out must be 16-byte aligned");
  const hipStream_t hs = static_cast<hipStream_t>(stream);
  if (debug_checks()) {
    st = debug_check_ranges(paged_kv, page_table, max_pages_per_seq, start_pos, lens, batch, INT32_MAX, max_len, 1,
                            total_tokens, false, hs);
    if (st != MBE_OK) return st;
  }
  mbe::KvQ8Params p = range_params(paged_kv, page_table, max_pages_per_seq, start_pos, lens, batch, max_len, total_tokens);
  p.k_out = static_cast<uint16_t *>(k_out);
  p.v_out = static_cast<uint16_t *>(v_out);
  const hipError_t e = mbe::launch_kv_read_q8(p, paged_kv->head_dim, paged_kv->format, hs);
  return e == hipSuccess ? MBE_OK : hip_error(e, "read-back launch");
}

mbe_status mbe_window_attention_q8(const void *q, const mbe_paged_kv_q8 *paged_kv, const int32_t *page_table,
                                   const int32_t *prefix_lens, const int32_t *window_lens, int32_t block_size,
                                   void *out, const mbe_attn_opts *opts) {
  mbe::AttnQ8Plan pl;
  mbe_status st = plan_attention(paged_kv, opts, block_size, &pl);
  if (st != MBE_OK) return st;
  const mbe_attn_opts *o = opts;
  if (o->batch == 0 || o->total_q == 0 || o->max_window_len == 0) return MBE_OK;
  st = check_pool_pointers(paged_kv);
  if (st != MBE_OK) return st;
  if (!q || !out || !page_table || !prefix_lens || !window_lens)
    return report(MBE_ERR_NULL_ARG, "q, out, page_table, prefix_lens and window_lens must be non-NULL");
  if (misaligned({q, out}, 16)) return report(MBE_ERR_BAD_SHAPE, "q and out must be 16-byte aligned");
  if (pl.bytes > 0) {
    if (!o->workspace) return report(MBE_ERR_WORKSPACE, "workspace of %zu bytes required", pl.bytes);
    if (o->workspace_bytes < pl.bytes)
      return report(MBE_ERR_WORKSPACE, "workspace %zu bytes < required %zu", o->workspace_bytes, pl.bytes);
    if (misaligned({o->workspace}, 256)) return report(MBE_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  }
  const hipStream_t hs = static_cast<hipStream_t>(o->stream);
  if (debug_checks()) {
    st = debug_check_ranges(paged_kv, page_table, o->max_pages_per_seq, prefix_lens, window_lens, o->batch,
                            o->max_prefix_len, o->max_window_len, block_size, o->total_q, true, hs);
    if (st != MBE_OK) return st;
  }
  mbe::AttnQ8Params p{};
  p.q = static_cast<const uint16_t *>(q);
  p.k_pages = static_cast<const uint8_t *>(paged_kv->k_pages);
  p.v_pages = static_cast<const uint8_t *>(paged_kv->v_pages);
  p.k_scales = paged_kv->k_scales;
  p.v_scales = paged_kv->v_scales;
  p.page_table = page_table;
  p.prefix_lens = prefix_lens;
  p.window_lens = window_lens;
  p.out = static_cast<uint16_t *>(out);
  char *ws = static_cast<char *>(o->workspace);
  p.notes = pl.bytes ? reinterpret_cast<int32_t *>(ws) : nullptr;
  p.part_o = pl.bytes ? reinterpret_cast<float *>(ws + pl.part_o_off) : nullptr;
  p.part_ml = pl.bytes ? reinterpret_cast<float *>(ws + pl.part_ml_off) : nullptr;
  p.batch = o->batch;
  p.num_q_heads = o->num_q_heads;
  p.num_kv_heads = paged_kv->num_kv_heads;
  p.group = o->num_q_heads / paged_kv->num_kv_heads;
  p.num_pages = paged_kv->num_pages;
  p.max_pages = o->max_pages_per_seq;
  p.block_size = block_size;
  p.total_q = o->total_q;
  p.max_prefix = o->max_prefix_len;
  p.max_window = o->max_window_len;
  p.causal = o->mask_mode == MBE_MASK_BLOCK_CAUSAL;
  const float scale = o->softmax_scale > 0.f ? o->softmax_scale : 1.0f / std::sqrt(static_cast<float>(paged_kv->head_dim));
  p.scale_log2 = scale * 1.4426950408889634f;
  p.block_flags = o->block_flags;
  p.flag_stride = o->max_window_len / block_size;
  p.gate = o->run_if_nonzero;
  p.wgs = pl.wgs;
  p.min_tiles = pl.min_tiles;
  p.start_tiles = pl.start_tiles;
  p.memory_tiles = pl.memory_tiles;
  p.join_tiles = pl.join_tiles;
  p.qtiles = pl.qtiles;
  p.split = pl.split;
  const hipError_t e = mbe::launch_attn_q8(p, pl, paged_kv->head_dim, paged_kv->format, hs);
  return e == hipSuccess ? MBE_OK : hip_error(e, "8-bit window attention launch");
}

size_t mbe_window_attention_q8_workspace_size(const mbe_paged_kv_q8 *paged_kv, const mbe_attn_opts *opts) {
  mbe::AttnQ8Plan pl;
  return plan_attention(paged_kv, opts, 1, &pl) == MBE_OK ? pl.bytes : static_cast<size_t>(-1);
}

mbe_status mbe_rotary(const void *q, void *q_out, int32_t num_q_heads, int64_t q_stride, int64_t q_out_stride,
                      const void *k, void *k_out, int32_t num_kv_heads, int64_t k_stride, int64_t k_out_stride,
                      int32_t head_dim, const int32_t *start_pos, const int32_t *lens, int32_t batch, int32_t max_len,
                      int32_t total_rows, const int64_t *turns, int32_t rot_dim, int32_t layout, float scale,
                      int32_t inverse, void *stream) {
  if (head_dim != 64 && head_dim != 128)
    return report(MBE_ERR_UNSUPPORTED, "head_dim %d: supported are 64 and 128", head_dim);
  if (rot_dim < 16 || rot_dim > head_dim || rot_dim % 16 != 0)
    return report(MBE_ERR_UNSUPPORTED, "rot_dim %d is not a multiple of 16 in [16, %d]", rot_dim, head_dim);
  if (layout != MBE_ROTARY_HALF && layout != MBE_ROTARY_INTERLEAVED)
    return report(MBE_ERR_UNSUPPORTED, "layout %d", layout);
  if (!std::isfinite(scale)) return report(MBE_ERR_BAD_VALUE, "scale is not finite");
  if (num_q_heads < 0 || num_kv_heads < 0 || num_q_heads > 65535 || num_kv_heads > 65535)
    return report(MBE_ERR_BAD_SHAPE, "num_q_heads %d / num_kv_heads %d outside [0, 65535]", num_q_heads, num_kv_heads);
  if (batch < 0 || batch > 65535) return report(MBE_ERR_BAD_SHAPE, "batch %d outside [0, 65535]", batch);
  if (max_len < 0 || total_rows < 0) return report(MBE_ERR_BAD_SHAPE, "negative max_len/total_rows");
  if (max_len > (1 << 27)) return report(MBE_ERR_BAD_SHAPE, "max_len %d is too large for one call", max_len);
  if (batch == 0 || max_len == 0 || total_rows == 0 || num_q_heads + num_kv_heads == 0) return MBE_OK;
  if (!start_pos || !lens || !turns) return report(MBE_ERR_NULL_ARG, "start_pos, lens and turns must be non-NULL");
  if ((num_q_heads > 0 && (!q || !q_out)) || (num_kv_heads > 0 && (!k || !k_out)))
    return report(MBE_ERR_NULL_ARG, "inputs and outputs with heads must be non-NULL");
  if (misaligned({q, q_out, k, k_out}, 16)) return report(MBE_ERR_BAD_SHAPE, "q, k and the outputs must be 16-byte aligned");
  if ((q_stride | q_out_stride | k_stride | k_out_stride) % 8 != 0)
    return report(MBE_ERR_BAD_SHAPE, "row strides must be multiples of 8 values");
  const int64_t qw = static_cast<int64_t>(num_q_heads) * head_dim, kw = static_cast<int64_t>(num_kv_heads) * head_dim;
  if (total_rows > 1 && (q_stride < qw || q_out_stride < qw || k_stride < kw || k_out_stride < kw))
    return report(MBE_ERR_BAD_SHAPE, "row strides smaller than a row");
  mbe::RotaryParams p{};
  p.q = static_cast<const uint16_t *>(q);
  p.k = static_cast<const uint16_t *>(k);
  p.q_out = static_cast<uint16_t *>(q_out);
  p.k_out = static_cast<uint16_t *>(k_out);
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.q_out_stride = q_out_stride;
  p.k_out_stride = k_out_stride;
  p.num_q_heads = num_q_heads;
  p.num_kv_heads = num_kv_heads;
  p.start_pos = start_pos;
  p.lens = lens;
  p.batch = batch;
  p.max_len = max_len;
  p.total_rows = total_rows;
  p.turns = reinterpret_cast<const uint64_t *>(turns);
  p.rot_dim = rot_dim;
  p.interleaved = layout == MBE_ROTARY_INTERLEAVED;
  p.inverse = inverse != 0;
  p.scale = scale;
  const hipError_t e = mbe::launch_rotary(p, head_dim, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? MBE_OK : hip_error(e, "rotation launch");
}

}  // extern "C"
