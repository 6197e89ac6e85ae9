// Quantising write into the 8-bit paged pools, and read-back, gfx950.
//
// A page of 16 tokens and one KV head is the unit of both: its values share
// one power-of-two scale s, the smallest with max|x| <= s * top (top = 448 for
// e4m3, 57344 for e5m2, both 1.75 * 2^n).  With |x| = 2^e (1 + m / 128) in bf16
// that is s = 2^(e - n + (m > 96)), read off the largest magnitude's bits, and
// x / s is exact, so the only rounding is the one to 8 bits.  An 8-bit float
// keeps its relative precision under any power of two: the scale costs at most
// one binade at the low end of the type's 2^15 (2^30) range, and a page whose
// scale grows under kept tokens moves them by an exponent shift.
//
// One wave per (page, head, K or V): the whole page (D = 128: 4 KB of bf16)
// sits in its registers between the maximum and the rounding, so every value
// is read once and nothing passes through LDS.  K rows are 16-byte chunks, 4
// rows to a load.  V pages are token-minor: a lane reads 4 bytes (two dims) of
// every token, 256 contiguous bytes per wave and load, and packs each dim's 16
// bytes in its own registers, where a transposition would otherwise need LDS.
// Both calls move 6 bytes a value pair and are bound by HBM for long ranges, by
// the chain lens -> page id -> scale for single tokens.  At 4 KV heads of 128 dims,
// 79000 tokens of 32 sequences written in 50 us (4.9 TB/s, what a large copy
// reaches), 151000 tokens read back in 84 us (5.6 TB/s); one token of each of 8
// sequences written in 4 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "q8.h"
#include "q8_device.h"

namespace mbe {
namespace {

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kMinScaleExp = -100, kMaxScaleExp = 120;

__device__ inline float bf_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ inline float bf_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ inline float exp2i(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// Four values to four bytes, lowest first.
template <int FMT>
__device__ inline uint32_t pack4(float a, float b, float c, float d) {
  int r = 0;
  if constexpr (FMT == MBE_Q8_E4M3) {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
  }
  return static_cast<uint32_t>(r);
}

template <int FMT>
__device__ inline void unpack4(uint32_t u, float *x) {
  f32x2 lo, hi;
  if constexpr (FMT == MBE_Q8_E4M3) {
    lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(u), false);
    hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(u), true);
  } else {
    lo = __builtin_amdgcn_cvt_pk_f32_bf8(static_cast<int>(u), false);
    hi = __builtin_amdgcn_cvt_pk_f32_bf8(static_cast<int>(u), true);
  }
  x[0] = lo[0];
  x[1] = lo[1];
  x[2] = hi[0];
  x[3] = hi[1];
}

// A kept dword of the page at the grown scale.  (An infinity, which only a
// pool written elsewhere can hold, becomes the largest finite value.)
template <int FMT>
__device__ inline uint32_t requantise(uint32_t u, float ratio) {
  constexpr float top = FMT == MBE_Q8_E4M3 ? 448.f : 57344.f;
  float x[4];
  unpack4<FMT>(u, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] *= ratio;
    x[i] = x[i] > top ? top : (x[i] < -top ? -top : x[i]);
  }
  return pack4<FMT>(x[0], x[1], x[2], x[3]);
}

// Byte mask of four mask bits.
__device__ inline uint32_t byte_mask(uint32_t bits) {
  return ((bits & 1u) | ((bits & 2u) << 7) | ((bits & 4u) << 14) | ((bits & 8u) << 21)) * 0xFFu;
}

// Magnitude bits of a wave's bf16 values, the largest in every lane.
__device__ inline uint32_t wave_max(u16x2 m) {
  uint32_t r = max(static_cast<uint32_t>(m[0]), static_cast<uint32_t>(m[1]));
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) r = max(r, static_cast<uint32_t>(__shfl_xor(static_cast<int>(r), o)));
  return r;
}

__device__ inline u16x2 magnitude(uint32_t u) { return __builtin_bit_cast(u16x2, u & 0x7FFF7FFFu); }

constexpr uint32_t kInfBits = 0x7F80;

// The same with infinities and NaN taken as 0.
__device__ inline u16x2 finite_magnitude(uint32_t u) {
  u16x2 m = magnitude(u);
  if (m[0] >= kInfBits) m[0] = 0;
  if (m[1] >= kInfBits) m[1] = 0;
  return m;
}

// Scale of a page whose largest finite magnitude has these bf16 bits.
template <int FMT>
__device__ inline float scale_of(uint32_t bits) {
  constexpr int top_exp = FMT == MBE_Q8_E4M3 ? 8 : 15;
  int e = static_cast<int>(bits >> 7) - 127 - top_exp + ((bits & 0x7F) > 96 ? 1 : 0);
  return exp2i(min(max(e, kMinScaleExp), kMaxScaleExp));
}

// x * inv; with SPECIAL, beyond the type's largest value (an infinity) that value.
template <int FMT, bool SPECIAL>
__device__ inline float scaled(float x, float inv) {
  constexpr float top = FMT == MBE_Q8_E4M3 ? 448.f : 57344.f;
  x *= inv;
  if constexpr (SPECIAL) x = x > top ? top : (x < -top ? -top : x);
  return x;
}

// Four dims of a token (two dwords of bf16), or one of the two dims of four
// tokens (four dwords), to four bytes.
template <int FMT, bool SPECIAL>
__device__ inline uint32_t pack_row(uint32_t a, uint32_t b, float inv) {
  return pack4<FMT>(scaled<FMT, SPECIAL>(bf_lo(a), inv), scaled<FMT, SPECIAL>(bf_hi(a), inv),
                    scaled<FMT, SPECIAL>(bf_lo(b), inv), scaled<FMT, SPECIAL>(bf_hi(b), inv));
}
template <int FMT, bool SPECIAL>
__device__ inline uint32_t pack_lo(const uint32_t *x, float inv) {
  return pack4<FMT>(scaled<FMT, SPECIAL>(bf_lo(x[0]), inv), scaled<FMT, SPECIAL>(bf_lo(x[1]), inv),
                    scaled<FMT, SPECIAL>(bf_lo(x[2]), inv), scaled<FMT, SPECIAL>(bf_lo(x[3]), inv));
}
template <int FMT, bool SPECIAL>
__device__ inline uint32_t pack_hi(const uint32_t *x, float inv) {
  return pack4<FMT>(scaled<FMT, SPECIAL>(bf_hi(x[0]), inv), scaled<FMT, SPECIAL>(bf_hi(x[1]), inv),
                    scaled<FMT, SPECIAL>(bf_hi(x[2]), inv), scaled<FMT, SPECIAL>(bf_hi(x[3]), inv));
}

// One wave's page of a ragged range: where it lies and which slots it covers.
struct PageItem {
  int g;               // KV head
  bool is_v;
  int64_t page;        // page index in the sequence's table row
  int64_t row;         // input/output row of the page's slot 0 (may be before the first row)
  int64_t pos;         // position of slot 0
  int64_t start, end;  // positions of the range
};

// False: the wave has nothing to do.
__device__ inline bool page_item(const KvQ8Params &p, PageItem *it) {
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x) * 4 + static_cast<int>(threadIdx.x >> 6));
  const int per_page = 2 * p.num_kv_heads;
  const int rel = wave / per_page;
  const int rem = wave - rel * per_page;
  const int b = blockIdx.y;
  const int len = min(max(p.lens[b], 0), p.max_len);
  if (len == 0) return false;
  it->g = rem >> 1;
  it->is_v = rem & 1;
  it->start = max(p.start_pos[b], 0);
  it->end = it->start + len;
  it->page = it->start / kPageSize + rel;
  it->pos = it->page * kPageSize;
  if (it->pos >= it->end) return false;
  it->row = rows_before(p.lens, b, p.max_len) + (it->pos - it->start);
  return true;
}

template <int D, int FMT>
__global__ __launch_bounds__(256) void kv_write_q8_kernel(KvQ8Params p) {
  PageItem it;
  if (!page_item(p, &it) || it.page >= p.max_pages) return;
  const int b = blockIdx.y;
  const int lane = threadIdx.x & 63;
  const int32_t pid = p.page_table[static_cast<int64_t>(b) * p.max_pages + it.page];
  if (pid < 0 || pid >= p.num_pages) return;
  const int64_t ph = static_cast<int64_t>(pid) * p.num_kv_heads + it.g;
  float *scale_at = (it.is_v ? p.v_scales : p.k_scales) + ph;
  const float old_scale = *scale_at;
  // new and kept slots (bit s for slot s): lane s tests slot s
  uint32_t wmask, kmask;
  {
    const int64_t pos = it.pos + (lane & 15);
    const int64_t t = pos - it.start;
    bool write = t >= 0 && pos < it.end && it.row + (lane & 15) < p.total_tokens;
    if (write && p.block_flags)
      write = p.block_flags[static_cast<int64_t>(b) * p.flag_stride + static_cast<int>(t) / p.block_size] != 0;
    const int64_t held = p.kv_lens ? max(it.start, static_cast<int64_t>(p.kv_lens[b])) : it.start;
    wmask = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(write)) & 0xFFFFu;
    kmask = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(!write && pos < held)) & 0xFFFFu;
  }
  if (wmask == 0) return;
  uint8_t *page = (it.is_v ? p.v_pages : p.k_pages) + ph * (kPageSize * D);
  const uint16_t *src = it.is_v ? p.v_new : p.k_new;
  constexpr int kWords = D / 8;       // dwords of bf16 a lane holds (16 tokens x D values / 64 lanes / 2)
  uint32_t x[kWords];
  // K: chunk of 8 dims of rows j * kRows + lane / kChunks;  V: two dims of kTok tokens
  constexpr int kChunks = D / 8, kRows = 64 / kChunks;
  constexpr int kPairs = D / 2, kTok = kWords;
  const int tok0 = (lane / kPairs) * kTok;
  if (!it.is_v) {
#pragma unroll
    for (int j = 0; j < kWords / 4; ++j) {
      const int slot = j * kRows + lane / kChunks;
      uint4 w = {0, 0, 0, 0};
      if ((wmask >> slot) & 1u)
        w = *reinterpret_cast<const uint4 *>(src + ((it.row + slot) * p.num_kv_heads + it.g) * D + (lane % kChunks) * 8);
      x[4 * j] = w.x;
      x[4 * j + 1] = w.y;
      x[4 * j + 2] = w.z;
      x[4 * j + 3] = w.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kTok; ++i) {
      const int slot = tok0 + i;
      x[i] = 0;
      if ((wmask >> slot) & 1u)
        x[i] = *reinterpret_cast<const uint32_t *>(src + ((it.row + slot) * p.num_kv_heads + it.g) * D + (lane % kPairs) * 2);
    }
  }
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < kWords; ++i) m = __builtin_elementwise_max(m, magnitude(x[i]));
  uint32_t top_bits = wave_max(m);
  const bool special = top_bits >= kInfBits;      // the same in every lane
  if (special) {
    m = {0, 0};
#pragma unroll
    for (int i = 0; i < kWords; ++i) m = __builtin_elementwise_max(m, finite_magnitude(x[i]));
    top_bits = wave_max(m);
  }
  float scale = scale_of<FMT>(top_bits);
  if (kmask) scale = fmaxf(scale, old_scale);
  const bool grew = kmask && scale > old_scale;
  const float inv = 1.0f / scale, ratio = old_scale / scale;
  auto store = [&](auto has_special) {
    constexpr bool S = decltype(has_special)::value;
    if (!it.is_v) {
#pragma unroll
      for (int j = 0; j < kWords / 4; ++j) {
        const int slot = j * kRows + lane / kChunks;
        uint2 *dst = reinterpret_cast<uint2 *>(page + slot * D + (lane % kChunks) * 8);
        if ((wmask >> slot) & 1u) {
          *dst = uint2{pack_row<FMT, S>(x[4 * j], x[4 * j + 1], inv), pack_row<FMT, S>(x[4 * j + 2], x[4 * j + 3], inv)};
        } else if (grew && ((kmask >> slot) & 1u)) {
          const uint2 w = *dst;
          *dst = uint2{requantise<FMT>(w.x, ratio), requantise<FMT>(w.y, ratio)};
        }
      }
      return;
    }
    uint32_t y[2][kTok / 4];      // the two dims' bytes, tokens in order
#pragma unroll
    for (int i = 0; i < kTok / 4; ++i) {
      y[0][i] = pack_lo<FMT, S>(x + 4 * i, inv);
      y[1][i] = pack_hi<FMT, S>(x + 4 * i, inv);
    }
    uint8_t *dst = page + (lane % kPairs) * 2 * kPageSize + tok0;
    if (wmask != 0xFFFFu) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < kTok / 4; ++i) {
          const uint32_t old = *reinterpret_cast<const uint32_t *>(dst + e * kPageSize + 4 * i);
          const uint32_t wm = byte_mask(wmask >> (tok0 + 4 * i)), km = byte_mask(kmask >> (tok0 + 4 * i));
          uint32_t r = old;
          if (grew) r = (old & ~km) | (requantise<FMT>(old, ratio) & km);
          y[e][i] = (y[e][i] & wm) | (r & ~wm);
        }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int i = 0; i < kTok / 4; i += 2)
        *reinterpret_cast<uint2 *>(dst + e * kPageSize + 4 * i) = uint2{y[e][i], y[e][i + 1]};
  };
  if (special) store(std::true_type{});
  else store(std::false_type{});
  if (lane == 0) *scale_at = scale;
}

template <int D, int FMT>
__global__ __launch_bounds__(256) void kv_read_q8_kernel(KvQ8Params p) {
  PageItem it;
  if (!page_item(p, &it)) return;
  const int b = blockIdx.y;
  const int lane = threadIdx.x & 63;
  int32_t pid = -1;
  if (it.page < p.max_pages) pid = p.page_table[static_cast<int64_t>(b) * p.max_pages + it.page];
  const bool valid = pid >= 0 && pid < p.num_pages;
  const int64_t ph = static_cast<int64_t>(valid ? pid : 0) * p.num_kv_heads + it.g;
  const float scale = (it.is_v ? p.v_scales : p.k_scales)[ph];
  const uint8_t *page = (it.is_v ? p.v_pages : p.k_pages) + ph * (kPageSize * D);
  // slots read: [s0, s1)
  const int s0 = static_cast<int>(max(it.start - it.pos, static_cast<int64_t>(0)));
  int s1 = static_cast<int>(min(it.end - it.pos, static_cast<int64_t>(kPageSize)));
  s1 = static_cast<int>(min(static_cast<int64_t>(s1), p.total_tokens - it.row));
  constexpr int kWords = D / 8;
  constexpr int kChunks = D / 8, kRows = 64 / kChunks;
  constexpr int kPairs = D / 2, kTok = kWords;
  auto pair = [](float lo, float hi) {
    bf16x2 r;
    r[0] = static_cast<__bf16>(lo);
    r[1] = static_cast<__bf16>(hi);
    return __builtin_bit_cast(uint32_t, r);
  };
  if (!it.is_v) {
    uint2 raw[kWords / 4];
#pragma unroll
    for (int j = 0; j < kWords / 4; ++j)
      raw[j] = *reinterpret_cast<const uint2 *>(page + (j * kRows + lane / kChunks) * D + (lane % kChunks) * 8);
#pragma unroll
    for (int j = 0; j < kWords / 4; ++j) {
      const int slot = j * kRows + lane / kChunks;
      if (slot < s0 || slot >= s1) continue;
      float f[8];
      unpack4<FMT>(raw[j].x, f);
      unpack4<FMT>(raw[j].y, f + 4);
      uint4 w = {pair(f[0] * scale, f[1] * scale), pair(f[2] * scale, f[3] * scale), pair(f[4] * scale, f[5] * scale),
                 pair(f[6] * scale, f[7] * scale)};
      if (!valid) w = {0, 0, 0, 0};
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, w), reinterpret_cast<u32x4 *>(p.k_out + ((it.row + slot) * p.num_kv_heads + it.g) * D + (lane % kChunks) * 8));
    }
  } else {
    const int tok0 = (lane / kPairs) * kTok;
    const uint8_t *at = page + (lane % kPairs) * 2 * kPageSize + tok0;
    float f[2][kTok];
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int i = 0; i < kTok; i += 8) {
        const uint2 raw = *reinterpret_cast<const uint2 *>(at + e * kPageSize + i);
        unpack4<FMT>(raw.x, &f[e][i]);
        unpack4<FMT>(raw.y, &f[e][i + 4]);
      }
#pragma unroll
    for (int i = 0; i < kTok; ++i) {
      const int slot = tok0 + i;
      if (slot < s0 || slot >= s1) continue;
      const uint32_t w = valid ? pair(f[0][i] * scale, f[1][i] * scale) : 0u;
      __builtin_nontemporal_store(w, reinterpret_cast<uint32_t *>(p.v_out + ((it.row + slot) * p.num_kv_heads + it.g) * D + (lane % kPairs) * 2));
    }
  }
}

// Waves of the longest sequence's pages, four to a workgroup; ceil(max_len /
// 16) + 1 pages (a range that starts inside a page).
dim3 page_grid(const KvQ8Params &p) {
  const int64_t pages = (static_cast<int64_t>(p.max_len) + kPageSize - 1) / kPageSize + 1;
  return dim3(static_cast<unsigned>((pages * 2 * p.num_kv_heads + 3) / 4), static_cast<unsigned>(p.batch));
}

}  // namespace

#define MBE_BY_FORM(kernel)                                                                          \
  do {                                                                                               \
    const dim3 grid = page_grid(p);                                                                  \
    if (head_dim == 128 && format == MBE_Q8_E4M3)                                                    \
      hipLaunchKernelGGL((kernel<128, MBE_Q8_E4M3>), grid, dim3(256), 0, stream, p);                 \
    else if (head_dim == 128)                                                                        \
      hipLaunchKernelGGL((kernel<128, MBE_Q8_E5M2>), grid, dim3(256), 0, stream, p);                 \
    else if (format == MBE_Q8_E4M3)                                                                  \
      hipLaunchKernelGGL((kernel<64, MBE_Q8_E4M3>), grid, dim3(256), 0, stream, p);                  \
    else                                                                                             \
      hipLaunchKernelGGL((kernel<64, MBE_Q8_E5M2>), grid, dim3(256), 0, stream, p);                  \
    return hipGetLastError();                                                                        \
  } while (0)

hipError_t launch_kv_write_q8(const KvQ8Params &p, int head_dim, int format, hipStream_t stream) {
  MBE_BY_FORM(kv_write_q8_kernel);
}

hipError_t launch_kv_read_q8(const KvQ8Params &p, int head_dim, int format, hipStream_t stream) {
  MBE_BY_FORM(kv_read_q8_kernel);
}

#undef MBE_BY_FORM

}  // namespace mbe
