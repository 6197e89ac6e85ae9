// Window attention over an 8-bit paged KV cache, gfx950.
//
//   S = c_page (K Q^T),  P = exp2(S - m),  O = (sum_key P V s_page) / sum_key P
//
// The cache's bytes feed the matrix cores as they are stored where they can.
// Q.K: v_mfma_f32_32x32x64_f8f6f4 multiplies 8-bit operands at twice bf16's
// rate.  K is one operand.  Q, a bf16 row with 8 significant bits, is the exact
// sum of two e4m3 numbers of 4 bits each: scaled by a power of two so that its
// largest magnitude is in [128, 256), hi = e4m3(x), lo = e4m3(x - hi).  (The
// sum is exact for |x| >= 2^-10 of that maximum, and within 2^-18 of it below.)
// Two 8-bit products cost what one in bf16 does, and K needs no conversion and
// half the registers and LDS bytes.  P.V: P has no bound that would suit 8
// bits, so V's bytes become bf16 (exactly), 16 keys of a dim at a time.
//
// Page scales cost nothing per value.  Key order within a matrix operand is
// free as long as both operands agree, and it is chosen so that an output lane
// holds the 16 keys of one page: row r of a 32-key block is key
// 16 ((r >> 2) & 1) + 4 (r >> 3) + (r & 3).  A lane's scale is then one number
// per page, folded with Q's and the softmax scale into the multiplier in front
// of exp2, and V's scale is added to the exponent as its logarithm (the row sum
// takes it out again, once per 16 keys).  The same order makes the output
// registers of Q.K the operand of P.V without a shuffle, and V's token-minor
// page rows (16 keys of a dim, 16 bytes) the other operand.
//
// The running maximum is raised only when a tile's exceeds it by 2^8: exact for
// any reference, and the accumulators are rescaled in a few tiles of a
// sequence instead of all.
//
// Work is dealt on the device, from the device lengths.  A unit is (sequence,
// KV head, tile of packed rows); all units' 64-key tiles in one line are cut
// into equal shares, one per workgroup.  A share that begins or ends inside a
// unit leaves a partial result (sum, maximum, accumulators), and a second
// kernel joins the parts of every unit that was cut, in the order of the
// shares: nothing depends on which workgroup is done first.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "q8.h"

namespace mbe {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kTile = 64;                   // keys of a tile: 4 pages
constexpr float kNegHuge = -1e30f;
constexpr float kLazy = 8.f;                // exponent headroom before the reference maximum is raised

__device__ inline int64_t wave_sum(int64_t x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// ------------------------------------------------------------ work dealing
struct Seq {
  int p, w;                 // prefix and window, clamped to the bounds
  int tiles, qtiles;        // key tiles, row tiles
};

template <int ROWS>
__device__ inline Seq seq_of(const AttnQ8Params &p, int b) {
  Seq s;
  s.p = min(max(p.prefix_lens[b], 0), p.max_prefix);
  s.w = min(max(p.window_lens[b], 0), p.max_window);
  s.tiles = static_cast<int>((static_cast<int64_t>(s.p) + s.w + kTile - 1) / kTile);
  s.qtiles = static_cast<int>((static_cast<int64_t>(s.w) * p.group + ROWS - 1) / ROWS);
  return s;
}

template <int ROWS>
__device__ inline int64_t seq_work(const AttnQ8Params &p, int b) {
  const Seq s = seq_of<ROWS>(p, b);
  return static_cast<int64_t>(s.tiles) * s.qtiles * p.num_kv_heads;
}

// All units' tiles.  Every lane of a wave must call.
template <int ROWS>
__device__ inline int64_t total_work(const AttnQ8Params &p) {
  int64_t sum = 0;
  for (int b = threadIdx.x & 63; b < p.batch; b += 64) sum += seq_work<ROWS>(p, b);
  return wave_sum(sum);
}

// First row of q of sequence b.
__device__ inline int64_t first_row(const AttnQ8Params &p, int b) {
  int64_t r = 0;
  for (int j = threadIdx.x & 63; j < b; j += 64) r += min(max(p.window_lens[j], 0), p.max_window);
  return wave_sum(r);
}

struct Unit {
  int b, g, qt;
  int64_t begin;            // its first tile in the line
  Seq s;
};

// The unit that holds tile t of the line (0 <= t < total_work).
template <int ROWS>
__device__ inline Unit unit_at(const AttnQ8Params &p, int64_t t) {
  const int lane = threadIdx.x & 63;
  int64_t base = 0;
  Unit u{};
  for (int b0 = 0; b0 < p.batch; b0 += 64) {
    const int b = b0 + lane;
    const int64_t own = b < p.batch ? seq_work<ROWS>(p, b) : 0;
    int64_t up = own;       // inclusive prefix sum across the lanes
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t v = __shfl_up(up, o);
      if (lane >= o) up += v;
    }
    const uint64_t past = __builtin_amdgcn_ballot_w64(base + up > t);
    if (past) {
      const int at = __builtin_ctzll(past);
      const int64_t start = base + __shfl(up - own, at);
      u.b = b0 + at;
      u.s = seq_of<ROWS>(p, u.b);
      const int64_t rel = t - start;
      const int unit = static_cast<int>(rel / u.s.tiles);
      u.g = unit / u.s.qtiles;
      u.qt = unit - u.g * u.s.qtiles;
      u.begin = start + static_cast<int64_t>(unit) * u.s.tiles;
      return u;
    }
    base += __shfl(up, 63);
  }
  return u;
}

__device__ inline int64_t share_of(const AttnQ8Params &p, int64_t total) {
  return max(static_cast<int64_t>(p.min_tiles), (total + p.wgs - 1) / p.wgs);
}

// Position i of packed row r within the window, and its q row / head.
__device__ inline bool row_wanted(const AttnQ8Params &p, const Unit &u, int64_t row0, int r) {
  if (r >= u.s.w * p.group) return false;
  const int i = r / p.group;
  if (row0 + i >= p.total_q) return false;
  return !p.block_flags || p.block_flags[static_cast<int64_t>(u.b) * p.flag_stride + i / p.block_size] != 0;
}

// ------------------------------------------------------------- the pieces
__device__ inline float across_halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float across_halves_add(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int FMT>
__device__ inline f32x16 mfma_qk(i32x8 k, i32x8 q, f32x16 c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, q, c, FMT == MBE_Q8_E5M2 ? 1 : 0, 0, 0, 0, 0, 0);
}

template <int FMT, bool HI>
__device__ inline uint32_t widen(uint32_t u) {       // two 8-bit values to bf16, exactly
  bf16x2 r;
  if constexpr (FMT == MBE_Q8_E4M3)
    r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(u), 1.0f, HI);
  else
    r = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(static_cast<int>(u), 1.0f, HI);
  return __builtin_bit_cast(uint32_t, r);
}

// Eight 8-bit keys of a dim to a bf16 operand.
template <int FMT>
__device__ inline bf16x8 widen8(uint32_t a, uint32_t b) {
  const uint4 w = {widen<FMT, false>(a), widen<FMT, true>(a), widen<FMT, false>(b), widen<FMT, true>(b)};
  return __builtin_bit_cast(bf16x8, w);
}

__device__ inline uint32_t pack2(float a, float b) {
  bf16x2 r;
  r[0] = static_cast<__bf16>(a);
  r[1] = static_cast<__bf16>(b);
  return __builtin_bit_cast(uint32_t, r);
}

// Q row of this lane as two 8-bit operands per 64 dims; returns the factor that
// undoes the row's scaling.  `src` null: a row of zeros.
template <int D>
__device__ inline float load_q(const uint16_t *src, i32x8 *hi, i32x8 *lo) {
  const int h = (threadIdx.x & 63) >> 5;
  uint4 raw[D / 64][4];
#pragma unroll
  for (int s = 0; s < D / 64; ++s)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      raw[s][j] = uint4{0, 0, 0, 0};
      if (src) raw[s][j] = *reinterpret_cast<const uint4 *>(src + s * 64 + h * 32 + j * 8);
    }
  float top = 0.f;
#pragma unroll
  for (int s = 0; s < D / 64; ++s)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t u[4] = {raw[s][j].x, raw[s][j].y, raw[s][j].z, raw[s][j].w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        top = fmaxf(top, fmaxf(fabsf(__uint_as_float(u[i] << 16)), fabsf(__uint_as_float(u[i] & 0xFFFF0000u))));
    }
  top = across_halves_max(top);
  // 2^(7 - e) for a maximum in [2^e, 2^(e+1)); e kept where both factors are normal numbers
  const int e = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -110), 120);
  const bool bad = !(top < __builtin_inff());       // an infinity: the row's result is NaN
  const float up = bad ? __builtin_nanf("") : __uint_as_float(static_cast<uint32_t>(127 + 7 - e) << 23);
#pragma unroll
  for (int s = 0; s < D / 64; ++s)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t u[4] = {raw[s][j].x, raw[s][j].y, raw[s][j].z, raw[s][j].w};
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const float a = __uint_as_float(u[i] << 16) * up, b = __uint_as_float(u[i] & 0xFFFF0000u) * up;
        const float c = __uint_as_float(u[i + 1] << 16) * up, d = __uint_as_float(u[i + 1] & 0xFFFF0000u) * up;
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
        const f32x2 ab = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), cd = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(a - ab[0], b - ab[1], 0, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(c - cd[0], d - cd[1], v, true);
        hi[s][j * 2 + i / 2] = w;
        lo[s][j * 2 + i / 2] = v;
      }
    }
  return __uint_as_float(static_cast<uint32_t>(127 - 7 + e) << 23);
}

__device__ inline int page_of(const AttnQ8Params &p, int b, int64_t slot) {
  const int64_t s = min(slot, static_cast<int64_t>(p.max_pages) - 1);
  return min(max(p.page_table[static_cast<int64_t>(b) * p.max_pages + s], 0), p.num_pages - 1);
}

// ------------------------------------------------- streaming kernel
// Units of 32 rows; the workgroup's four waves take key tiles in turn, each
// straight from HBM into its registers, and join their results in LDS.
constexpr int kStreamRows = 32;
constexpr int kStreamWaves = 4;

template <int D, int FMT>
struct StreamTile {
  uint4 k[2][D / 32];       // [32-key block][16-byte chunk of the lane's key]
  uint4 v[2][D / 32];       // [32-key block][32-dim block]: 16 keys of the lane's dim
  float ks[2], vs[2];       // scales of the lane's page of each block
  int pid;                  // page (lane & 3) of the tile
};

template <int D, int FMT>
__global__ __launch_bounds__(kStreamWaves * 64, 2) void attn_q8_stream_kernel(AttnQ8Params p) {
  constexpr int NB = D / 32;              // 32-dim blocks
  constexpr int NS = D / 64;              // 64-dim contraction steps
  constexpr int kStride = D + 4;          // floats of a row in LDS
  __shared__ __align__(16) float o_lds[kStreamWaves][kStreamRows][kStride];
  __shared__ float ml_lds[kStreamWaves][kStreamRows][2];
  if (p.gate && *p.gate == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 31, h = lane >> 5;
  const int kslot = 4 * (col >> 3) + (col & 3);       // the lane's key (K operand): slot in its page
  const int kpage = (col >> 2) & 1;                   // and page of the 32-key block

  int64_t t0, t1, share = 0;
  Unit u{};
  if (p.split) {
    const int64_t total = total_work<kStreamRows>(p);
    share = share_of(p, total);
    t0 = share * blockIdx.x;
    t1 = min(t0 + share, total);
    if (t0 >= t1) return;
    u = unit_at<kStreamRows>(p, t0);
  } else {
    const int qt = static_cast<int>(blockIdx.x) % p.qtiles, rest = static_cast<int>(blockIdx.x) / p.qtiles;
    u.b = rest / p.num_kv_heads;
    u.g = rest - u.b * p.num_kv_heads;
    u.qt = qt;
    u.s = seq_of<kStreamRows>(p, u.b);
    u.begin = 0;
    if (qt >= u.s.qtiles) return;
    t0 = 0;
    t1 = u.s.tiles;
  }
  int64_t t = t0;
  while (true) {
    const int ta = static_cast<int>(t - u.begin);
    const int tb = static_cast<int>(min(t1 - u.begin, static_cast<int64_t>(u.s.tiles)));
    const int64_t row0 = first_row(p, u.b);
    const int n = u.s.p + u.s.w;
    const int r = u.qt * kStreamRows + col;           // packed row of this lane
    const bool wanted = row_wanted(p, u, row0, r);
    const bool any = __builtin_amdgcn_ballot_w64(wanted) != 0;      // the same in every wave
    if (any) {
      const int wi = r / p.group;
      const int seen = !wanted ? 0 : (p.causal ? min(n, u.s.p + (wi / p.block_size + 1) * p.block_size) : n);
      i32x8 qh[NS], ql[NS];
      const float qs = load_q<D>(wanted ? p.q + ((row0 + wi) * p.num_q_heads + u.g * p.group + r % p.group) * D : nullptr, qh, ql);
      const float cq = qs * p.scale_log2;

      f32x16 acc[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) acc[i] = f32x16{};
      float m = kNegHuge, l = 0.f;

      auto pages_of_tile = [&](int tile) { return page_of(p, u.b, static_cast<int64_t>(tile) * 4 + (lane & 3)); };
      auto load_k = [&](StreamTile<D, FMT> &x) {
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          const int a = __builtin_amdgcn_readlane(x.pid, 2 * blk), b = __builtin_amdgcn_readlane(x.pid, 2 * blk + 1);
          const int64_t ph = static_cast<int64_t>(kpage ? b : a) * p.num_kv_heads + u.g;
          const uint8_t *at = p.k_pages + (ph * kPageSize + kslot) * D + h * 32;
#pragma unroll
          for (int j = 0; j < NB; ++j) x.k[blk][j] = *reinterpret_cast<const uint4 *>(at + (j >> 1) * 64 + (j & 1) * 16);
        }
      };
      auto load_v = [&](StreamTile<D, FMT> &x) {
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          const int a = __builtin_amdgcn_readlane(x.pid, 2 * blk), b = __builtin_amdgcn_readlane(x.pid, 2 * blk + 1);
          const int64_t ph = static_cast<int64_t>(h ? b : a) * p.num_kv_heads + u.g;
          const uint8_t *at = p.v_pages + (ph * D + col) * kPageSize;
#pragma unroll
          for (int j = 0; j < NB; ++j) x.v[blk][j] = *reinterpret_cast<const uint4 *>(at + j * 32 * kPageSize);
          x.ks[blk] = p.k_scales[ph];
          x.vs[blk] = p.v_scales[ph];
        }
      };

      for (int tile = ta + wave; tile < tb; tile += kStreamWaves) {
        StreamTile<D, FMT> x;
        x.pid = pages_of_tile(tile);
        load_k(x);
        load_v(x);
        f32x16 s[2];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          s[blk] = f32x16{};
#pragma unroll
          for (int st = 0; st < NS; ++st) {
            i32x8 k;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              const uint4 c = x.k[blk][2 * st + w];
              k[4 * w] = c.x;
              k[4 * w + 1] = c.y;
              k[4 * w + 2] = c.z;
              k[4 * w + 3] = c.w;
            }
            s[blk] = mfma_qk<FMT>(k, qh[st], s[blk]);
            s[blk] = mfma_qk<FMT>(k, ql[st], s[blk]);
          }
        }
        const int key0 = tile * kTile + 16 * h;      // the lane's first key (block 0)
        // (covered pages have positive finite scales; the others hold anything)
        float c[2], lv[2], iv[2];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          c[blk] = fmaxf(x.ks[blk] * cq, 1.17549435e-38f);
          const float vs = fminf(fmaxf(x.vs[blk], 0x1p-100f), 0x1p100f);
          lv[blk] = __builtin_amdgcn_logf(vs);
          iv[blk] = __builtin_amdgcn_rcpf(vs);
        }
        const bool whole = tile * kTile + kTile <= u.s.p;      // every row sees every key
        if (!whole) {
#pragma unroll
          for (int blk = 0; blk < 2; ++blk) {
            const int left = seen - (key0 + 32 * blk);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[blk][i] = i < left ? s[blk][i] : -__builtin_inff();
            // slots behind the last token may hold NaN codes: 0 x NaN is NaN
            const int held = n - (key0 + 32 * blk);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
              uint32_t *d = reinterpret_cast<uint32_t *>(&x.v[blk][j]);
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                const int nb = min(max(held - 4 * w, 0), 4);
                d[w] = nb == 4 ? d[w] : d[w] & ((1u << (8 * nb)) - 1u);
              }
            }
          }
        }
        float mt = kNegHuge;
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          float mb = s[blk][0];
#pragma unroll
          for (int i = 1; i < 16; ++i) mb = fmaxf(mb, s[blk][i]);
          mt = fmaxf(mt, mb * c[blk]);
        }
        mt = across_halves_max(mt);
        if (__builtin_amdgcn_ballot_w64(mt > m + kLazy)) {
          const float mn = fmaxf(m, mt);
          const float a = __builtin_amdgcn_exp2f(m - mn);
          m = mn;
          l *= a;
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[j][i] *= a;
        }
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          const float off = lv[blk] - m;
          float sum = 0.f;
          uint32_t pk[8];
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float a = __builtin_amdgcn_exp2f(fmaf(s[blk][i], c[blk], off));
            const float b = __builtin_amdgcn_exp2f(fmaf(s[blk][i + 1], c[blk], off));
            sum += a;
            sum += b;
            pk[i / 2] = pack2(a, b);
          }
          l = fmaf(sum, iv[blk], l);
#pragma unroll
          for (int j2 = 0; j2 < 2; ++j2) {
            const uint4 pw = {pk[4 * j2], pk[4 * j2 + 1], pk[4 * j2 + 2], pk[4 * j2 + 3]};
            const bf16x8 pb = __builtin_bit_cast(bf16x8, pw);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
              const uint32_t *d = reinterpret_cast<const uint32_t *>(&x.v[blk][j]);
              acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8<FMT>(d[2 * j2], d[2 * j2 + 1]), pb, acc[j], 0, 0, 0);
            }
          }
        }
      }
      l = across_halves_add(l);
      if (h == 0) {
        ml_lds[wave][col][0] = m;
        ml_lds[wave][col][1] = l;
      }
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const f32x4 w = {acc[j][4 * a], acc[j][4 * a + 1], acc[j][4 * a + 2], acc[j][4 * a + 3]};
          *reinterpret_cast<f32x4 *>(&o_lds[wave][col][j * 32 + 8 * a + 4 * h]) = w;
        }
      __syncthreads();
      // join the waves: eight threads to a row, D / 8 dims each
      const int jr = threadIdx.x >> 3, part = threadIdx.x & 7;
      float mm = kNegHuge;
#pragma unroll
      for (int w = 0; w < kStreamWaves; ++w) mm = fmaxf(mm, ml_lds[w][jr][0]);
      float ll = 0.f, wt[kStreamWaves];
#pragma unroll
      for (int w = 0; w < kStreamWaves; ++w) {
        wt[w] = __builtin_amdgcn_exp2f(ml_lds[w][jr][0] - mm);
        ll += wt[w] * ml_lds[w][jr][1];
      }
      const int jrow = u.qt * kStreamRows + jr;
      const bool cut = ta > 0 || tb < u.s.tiles;
      const float inv = cut ? 1.f : 1.f / ll;
      f32x4 o[D / 32];
#pragma unroll
      for (int q = 0; q < D / 32; ++q) {
        o[q] = f32x4{};
#pragma unroll
        for (int w = 0; w < kStreamWaves; ++w) {
          const f32x4 v = *reinterpret_cast<const f32x4 *>(&o_lds[w][jr][part * (D / 8) + 4 * q]);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[q][i] += wt[w] * v[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) o[q][i] *= inv;
      }
      if (cut) {
        const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (t == t0 ? 0 : 1);
        float *dst = p.part_o + (slot * kStreamRows + jr) * D + part * (D / 8);
#pragma unroll
        for (int q = 0; q < D / 32; ++q) *reinterpret_cast<f32x4 *>(dst + 4 * q) = o[q];
        if (part == 0) {
          p.part_ml[(slot * kStreamRows + jr) * 2] = mm;
          p.part_ml[(slot * kStreamRows + jr) * 2 + 1] = ll;
        }
      } else if (row_wanted(p, u, row0, jrow)) {
        uint16_t *dst = p.out + ((row0 + jrow / p.group) * p.num_q_heads + u.g * p.group + jrow % p.group) * D + part * (D / 8);
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
          const uint2 w = {pack2(o[q][0], o[q][1]), pack2(o[q][2], o[q][3])};
          *reinterpret_cast<uint2 *>(dst + 4 * q) = w;
        }
      }
      __syncthreads();
    }
    t = u.begin + tb;
    if (t >= t1) return;
    u = unit_at<kStreamRows>(p, t);
  }
}

// ------------------------------------------------------------- the join
// Workgroup x looks at the border between shares x and x + 1.  Where it is the
// first border inside a unit, the workgroup joins that unit's parts; y takes
// eight rows each.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void attn_q8_join_kernel(AttnQ8Params p) {
  if (p.gate && *p.gate == 0) return;
  const int64_t total = total_work<ROWS>(p);
  const int64_t share = share_of(p, total);
  const int64_t border = share * (static_cast<int64_t>(blockIdx.x) + 1);
  if (border >= total) return;
  const Unit u = unit_at<ROWS>(p, border);
  if (u.begin >= border || border - share > u.begin) return;      // at the unit's start, or not its first border
  const int64_t row0 = first_row(p, u.b);
  constexpr int kLanes = D / 4;                     // lanes of a row, 4 dims each
  const int r_in = static_cast<int>(blockIdx.y) * (256 / kLanes) + static_cast<int>(threadIdx.x) / kLanes;
  const int d = (static_cast<int>(threadIdx.x) % kLanes) * 4;
  const int r = u.qt * ROWS + r_in;
  if (!row_wanted(p, u, row0, r)) return;
  const int64_t end = u.begin + u.s.tiles;
  const int64_t w0 = u.begin / share, w1 = (end - 1) / share;
  float m = kNegHuge, l = 0.f;
  f32x4 o = {};
  for (int64_t w = w0; w <= w1; ++w) {
    // the share that the unit begins in holds it second, unless it begins there too
    const int64_t slot = 2 * w + (w == w0 && u.begin != w * share ? 1 : 0);
    const float pm = p.part_ml[(slot * ROWS + r_in) * 2], pl = p.part_ml[(slot * ROWS + r_in) * 2 + 1];
    const f32x4 v = *reinterpret_cast<const f32x4 *>(p.part_o + (slot * ROWS + r_in) * D + d);
    const float mn = fmaxf(m, pm);
    const float a = __builtin_amdgcn_exp2f(m - mn), b = __builtin_amdgcn_exp2f(pm - mn);
    m = mn;
    l = l * a + pl * b;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = o[i] * a + v[i] * b;
  }
  const float inv = 1.f / l;
  uint16_t *dst = p.out + ((row0 + r / p.group) * p.num_q_heads + u.g * p.group + r % p.group) * D + d;
  const uint2 w = {pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv)};
  *reinterpret_cast<uint2 *>(dst) = w;
}

template <int D, int FMT>
hipError_t launch(const AttnQ8Params &p, const AttnQ8Plan &plan, hipStream_t stream) {
  hipLaunchKernelGGL((attn_q8_stream_kernel<D, FMT>), dim3(static_cast<unsigned>(plan.wgs)), dim3(kStreamWaves * 64), 0,
                     stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !plan.split || plan.wgs < 2) return e;
  const int rows = 256 / (D / 4);
  hipLaunchKernelGGL((attn_q8_join_kernel<D, kStreamRows>), dim3(static_cast<unsigned>(plan.wgs - 1), kStreamRows / rows),
                     dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_q8(const AttnQ8Params &p, const AttnQ8Plan &plan, int head_dim, int format, hipStream_t stream) {
  if (head_dim == 128)
    return format == MBE_Q8_E4M3 ? launch<128, MBE_Q8_E4M3>(p, plan, stream) : launch<128, MBE_Q8_E5M2>(p, plan, stream);
  return format == MBE_Q8_E4M3 ? launch<64, MBE_Q8_E4M3>(p, plan, stream) : launch<64, MBE_Q8_E5M2>(p, plan, stream);
}

}  // namespace mbe
