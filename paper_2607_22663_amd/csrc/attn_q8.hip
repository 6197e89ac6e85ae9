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
// The softmax's reference exponent is raised only when a tile's sum overflows a
// limit (softmax_tile), in a few tiles of a sequence instead of all.
//
// Work is dealt on the device, from the device lengths.  A unit is (sequence,
// KV head, tile of packed rows); all units' 64-key tiles in one line are cut
// into equal shares, one per workgroup.  A share that begins or ends inside a
// unit leaves a partial result (sum, maximum, accumulators), and a second
// kernel joins the parts of every unit that was cut, in the order of the
// shares: nothing depends on which workgroup is done first.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "q8.h"
#include "q8_device.h"

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

// ------------------------------------------------------------ work dealing
// A workgroup's piece of a unit: tiles [ta, tb) of tile range [0, tiles) of row
// tile qt of KV head g of sequence b, whose window starts at row row0 of q.
struct Piece {
  int b, g, qt, p, w, row0, ta, tb, tiles;
};

// The line of all units' tiles, cut into shares.
//   Few tiles: units are padded to whole shares of min_tiles, so that a workgroup
//   never has pieces of two units.
//   Units alike, and no more than workgroups: a unit each, where the longest takes
//   no longer than equal shares, or than the memory needs for all, and a join.
//   Otherwise every workgroup takes an equal share, across units.  There a unit has
//   start_tiles places before its tiles, the time that beginning one takes.
// (The launch bounds the line to 32 bits.)
template <int ROWS>
struct Deal {
  const AttnQ8Params &p;
  uint32_t share, at, end;      // this workgroup's part of the line: [at, end)
  uint32_t begin, length;       // the unit at hand in the line
  uint32_t pieces;              // of this workgroup before the one at hand
  bool padded;

  __device__ uint32_t starts() const { return padded ? 0 : p.start_tiles; }
  __device__ uint32_t whole(uint32_t tiles) const {
    return padded ? (tiles + share - 1) / share * share : tiles + p.start_tiles;
  }
  // The lane's sequence b: lengths within the bounds (0 behind the batch).
  struct Lens {
    int p, w;
  };
  __device__ Lens lens_of(int b) const {
    Lens s = {0, 0};
    if (b < p.batch) s = {p.prefix_lens[b], p.window_lens[b]};
    return {min(max(s.p, 0), p.max_prefix), min(max(s.w, 0), p.max_window)};
  }
  __device__ uint32_t tiles_of(Lens s) const { return (static_cast<uint32_t>(s.p) + s.w + kTile - 1) / kTile; }
  __device__ uint32_t units_of(Lens s) const {
    return (static_cast<uint32_t>(s.w) * p.group + ROWS - 1) / ROWS * p.num_kv_heads;
  }

  // Its first piece; false: it has none.
  __device__ bool start(Piece &u) {
    const int lane = threadIdx.x & 63;
    if (!p.split) {        // a whole unit each
      const int rest = static_cast<int>(blockIdx.x) / p.qtiles;
      u.qt = static_cast<int>(blockIdx.x) - rest * p.qtiles;
      u.b = rest / p.num_kv_heads;
      u.g = rest - u.b * p.num_kv_heads;
      uint32_t rows = 0, units = 0;
      for (int b0 = 0; b0 <= u.b; b0 += 64) {
        const Lens s = lens_of(b0 + lane);
        const uint32_t up = scan_lanes(s.w);
        if (u.b < b0 + 64) {
          const int l = u.b - b0;
          u.p = lane_value(s.p, l);
          u.w = lane_value(s.w, l);
          u.tiles = lane_value(tiles_of(s), l);
          u.row0 = rows + lane_value(up, l) - u.w;
          units = lane_value(units_of(s), l);
        }
        rows += lane_value(up, 63);
      }
      u.ta = 0;
      u.tb = u.tiles;
      at = end = pieces = 0;
      return u.qt * p.num_kv_heads < static_cast<int>(units);
    }
    uint32_t tight = 0, loose = 0, count = 0, longest = 0;
    padded = true;
    share = p.min_tiles;
    Lens s{};
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      s = lens_of(b0 + lane);
      const uint32_t tiles = tiles_of(s), units = units_of(s);
      tight += lane_value(scan_lanes((tiles + p.start_tiles) * units), 63);
      loose += lane_value(scan_lanes(whole(tiles) / share * units), 63);     // in shares
      count += lane_value(scan_lanes(units), 63);
      longest = max(longest, lane_value(max_lanes(units ? tiles : 0), 63));
    }
    padded = loose <= static_cast<uint32_t>(p.wgs);
    const uint32_t even = max(share, padded ? 0 : (tight + p.wgs - 1) / p.wgs);
    if (count <= static_cast<uint32_t>(p.wgs) && longest <= max(even, tight / p.memory_tiles) + p.join_tiles) {
      padded = true;
      share = longest;
      loose = count;
    } else if (!padded) {
      share = even;
    }
    const uint32_t total = padded ? loose * share : tight;
    at = share * blockIdx.x;
    end = min(at + share, total);
    pieces = 0;
    if (total == 0 || blockIdx.x > (total - 1) / share) return false;      // (share > 0 where total is)
    if (p.batch <= 64) {
      uint32_t base = 0, rows = 0;
      in_chunk(u, 0, s, base, rows);
    } else {
      piece(u);
    }
    return u.ta < u.tb || next(u);
  }

  // Whether `at` lies in the 64 sequences from b0 on (the lanes hold their lengths);
  // the piece there.  base, rows: places and rows before them, moved past them if not.
  __device__ bool in_chunk(Piece &u, int b0, Lens s, uint32_t &base, uint32_t &rows) {
    const uint32_t tiles = tiles_of(s), units = units_of(s);
    const uint32_t own = whole(tiles) * units, up = scan_lanes(own), wup = scan_lanes(s.w);
    const uint64_t past = __builtin_amdgcn_ballot_w64(base + up > at);
    if (!past) {
      base += lane_value(up, 63);
      rows += lane_value(wup, 63);
      return false;
    }
    const int l = __builtin_ctzll(past);
    u.b = b0 + l;
    u.p = lane_value(s.p, l);
    u.w = lane_value(s.w, l);
    u.tiles = lane_value(tiles, l);
    u.row0 = rows + lane_value(wup, l) - u.w;
    const uint32_t from = base + lane_value(up, l) - lane_value(own, l);
    const uint32_t qtiles = lane_value(units, l) / p.num_kv_heads;
    length = whole(u.tiles);
    const uint32_t unit = (at - from) / length;
    u.g = unit / qtiles;
    u.qt = unit - u.g * qtiles;
    begin = from + unit * length;
    const uint32_t first = begin + starts();       // its tile 0
    u.ta = at > first ? at - first : 0;
    u.tb = min(static_cast<uint32_t>(u.tiles), end > first ? end - first : 0);
    return true;
  }

  // The piece at `at`.
  __device__ void piece(Piece &u) {
    uint32_t base = 0, rows = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64)
      if (in_chunk(u, b0, lens_of(b0 + static_cast<int>(threadIdx.x & 63)), base, rows)) return;
  }

  // The next piece of its share; false: it has no more.  (A share may end before a
  // unit's first tile.)
  __device__ bool next(Piece &u) {
    if (!p.split || padded) return false;
    if (u.ta < u.tb) ++pieces;
    at = begin + length;
    if (at >= end) return false;
    piece(u);
    return u.ta < u.tb;
  }

  // Slot of the partial result of the piece at hand: a share has at most two, its
  // first piece and its last.
  __device__ int64_t slot() const { return 2 * static_cast<int64_t>(blockIdx.x) + (pieces == 0 ? 0 : 1); }
};

// What the join kernel is told by the workgroup with a unit's second part: the
// parts lie in slots slot, 2 wg, 2 wg + 2, ...
struct JoinNote {
  int32_t parts;            // 0: nothing to join here
  int32_t b, g, qt, w, row0, slot, unused;
};

template <int ROWS>
__device__ inline void leave_note(const AttnQ8Params &p, const Deal<ROWS> &d, const Piece &u, bool any) {
  if (!p.split || threadIdx.x != 0) return;
  JoinNote n{};
  const uint32_t wg = blockIdx.x;
  if (any && u.ta > 0) {
    // the shares with the unit's first and last tile; the first holds it second
    // where the share begins in the unit before
    const uint32_t w0 = (d.begin + d.starts()) / d.share, w1 = (d.begin + d.length - 1) / d.share;
    if (wg == w0 + 1) {
      n.parts = static_cast<int32_t>(w1 - w0 + 1);
      n.b = u.b;
      n.g = u.g;
      n.qt = u.qt;
      n.w = u.w;
      n.row0 = u.row0;
      n.slot = static_cast<int32_t>(2 * w0 + (w0 * d.share < d.begin ? 1 : 0));
    }
  }
  *reinterpret_cast<JoinNote *>(p.notes + 8 * static_cast<int64_t>(wg)) = n;
}

// Whether packed row r of the sequence's KV head is one that the call computes.
__device__ inline bool row_wanted(const AttnQ8Params &p, int b, int w, int row0, int r) {
  if (r >= w * p.group) return false;
  const int i = r / p.group;
  const int64_t row = static_cast<int64_t>(row0) + i;
  if (row < 0 || row >= p.total_q) return false;      // (lengths that do not fit the rows)
  return !p.block_flags || p.block_flags[static_cast<int64_t>(b) * p.flag_stride + i / p.block_size] != 0;
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

// This lane's half of a row of Q, as it is (asked for early, turned into operands
// while the first keys are on their way).  `src` null: zeros.
template <int D>
struct QRow {
  uint4 v[D / 64][4];
  __device__ void load(const uint16_t *src) {
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int s = 0; s < D / 64; ++s)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[s][j] = uint4{0, 0, 0, 0};
        if (src) v[s][j] = *reinterpret_cast<const uint4 *>(src + s * 64 + h * 32 + j * 8);
      }
  }
};

// Q row of this lane as two 8-bit operands per 64 dims; returns the factor that
// undoes the row's scaling.
template <int D>
__device__ inline float make_q(const QRow<D> &q, i32x8 *hi, i32x8 *lo) {
  const auto &raw = q.v;
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

// Entry of the page table, as it is: where it is looked at right after the load,
// the wave waits for every load in flight, so its clamping is left to its use.
__device__ inline int page_entry(const AttnQ8Params &p, int b, int64_t slot) {
  const int64_t s = min(slot, static_cast<int64_t>(p.max_pages) - 1);
  return p.page_table[static_cast<int64_t>(b) * p.max_pages + s];
}
__device__ inline int clamp_page(const AttnQ8Params &p, int entry) { return min(max(entry, 0), p.num_pages - 1); }

// A 32-key block's softmax: s (scores before scaling, -inf where masked) of the
// lane's 16 keys of one page to packed probabilities times V's scale, relative to
// the reference exponent m; l and acc follow a raised m.
//
// Optimistic: the probabilities are computed against the old reference, and only
// where a lane's sum exceeds 2^16 (or is no number) does the wave take the
// block's maximum, raise the reference and compute them again.  Any reference is
// exact, so the result is off by no more than fp32's rounding, and a block costs
// no maximum (of 16 values and across lanes).
constexpr float kSumLimit = 65536.f;

// Raises m to the block's maximum; the sum and the accumulators follow.
template <int NB>
__device__ inline void raise_reference(const f32x16 &s, float c, float &m, float &l, f32x16 *acc) {
  float mt = s[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) mt = fmaxf(mt, s[i]);
  mt = across_halves_max(fmaxf(kNegHuge, mt * c));
  const float mn = fmaxf(m, mt);
  const float a = __builtin_amdgcn_exp2f(m - mn);
  m = mn;
  l *= a;
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[j][i] *= a;
}

template <int NB>
__device__ inline void softmax_block(const f32x16 &s, float c, float lv, float iv, float &m, float &l, f32x16 *acc, bf16x8 *pb) {
  float sum;
  auto exps = [&]() {
    const float off = lv - m;
    uint32_t pk[8];
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float a = __builtin_amdgcn_exp2f(fmaf(s[i], c, off)), b = __builtin_amdgcn_exp2f(fmaf(s[i + 1], c, off));
      t += a;
      t += b;
      pk[i / 2] = pack2(a, b);
    }
    sum = t * iv;
    pb[0] = __builtin_bit_cast(bf16x8, (uint4{pk[0], pk[1], pk[2], pk[3]}));
    pb[1] = __builtin_bit_cast(bf16x8, (uint4{pk[4], pk[5], pk[6], pk[7]}));
  };
  exps();
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= kSumLimit)) != 0, 0)) {
    raise_reference<NB>(s, c, m, l, acc);
    exps();
  }
  l += sum;
}

// Per page: factor of the scores apart from the row's, logarithm and reciprocal
// of V's scale.  (Covered pages have positive finite scales; others hold anything.)
__device__ inline float k_factor(float ks, float cq) { return fmaxf(ks * cq, 1.17549435e-38f); }
__device__ inline float v_factor(float vs) { return fminf(fmaxf(vs, 0x1p-100f), 0x1p100f); }

// Bytes of a 16-byte row of V, 16 keys, from the `held`th key on to zero: slots
// behind the last token may hold NaN codes, and 0 x NaN is NaN.
__device__ inline uint32_t keys_of(uint32_t d, int held) {       // of 4 keys
  const int nb = min(max(held, 0), 4);
  return nb == 4 ? d : d & ((1u << (8 * nb)) - 1u);
}
__device__ inline uint4 zero_behind(uint4 v, int held) {
  return uint4{keys_of(v.x, held), keys_of(v.y, held - 4), keys_of(v.z, held - 8), keys_of(v.w, held - 12)};
}

__device__ inline i32x8 operand(uint4 a, uint4 b) {
  i32x8 k;
  k[0] = a.x;
  k[1] = a.y;
  k[2] = a.z;
  k[3] = a.w;
  k[4] = b.x;
  k[5] = b.y;
  k[6] = b.z;
  k[7] = b.w;
  return k;
}

// ------------------------------------------------- streaming kernel
// Units of 32 rows; the workgroup's four waves take key tiles in turn, each
// straight from HBM into its registers, and join their results in LDS.  A tile's
// K and V registers are loaded again for the wave's next tile right after their
// last use, so that 8 to 16 KB a wave are always on their way.  Bound by HBM (2 D
// bytes a key, and few operations): one token of 32 sequences of 65536 keys, 4 KV
// heads of 128 dims, 355 us, 6.05 TB/s; of 1000 to 8192 keys 34 us, 4.5 TB/s, of
// which about 5 are the first loads' round trips (length, page, K) and the join in
// LDS.
constexpr int kStreamRows = 32;
constexpr int kStreamWaves = 4;

template <int D, int FMT>
__global__ __launch_bounds__(kStreamWaves * 64, 2) void attn_q8_stream_kernel(AttnQ8Params p) {
  constexpr int NB = D / 32;              // 32-dim blocks
  constexpr int NS = D / 64;              // 64-dim contraction steps
  constexpr int kStride = D + 4;          // floats of a row in LDS
  __shared__ __align__(16) float o_lds[kStreamWaves][kStreamRows][kStride];
  __shared__ float ml_lds[kStreamWaves][kStreamRows][2];
  if (p.gate && *p.gate == 0) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, h = lane >> 5;
  const int kpage = (col >> 2) & 1;                   // the lane's key (K operand): its page of the block,
  const int k_src = (4 * (col >> 3) + (col & 3)) * D + h * 32;     // and byte in the page

  Deal<kStreamRows> deal{p};
  Piece u;
  const bool work = deal.start(u);
  leave_note(p, deal, u, work);
  if (!work) return;
  do {
    const int ta = u.ta, tb = u.tb;
    const int64_t row0 = u.row0;
    const int n = u.p + u.w;
    const int r = u.qt * kStreamRows + col;           // packed row of this lane
    const bool wanted = row_wanted(p, u.b, u.w, u.row0, r);
    const bool any = __builtin_amdgcn_ballot_w64(wanted) != 0;      // the same in every wave
    if (any) {
      const int wi = r / p.group;
      const int seen = !wanted ? 0 : (p.causal ? min(n, u.p + (wi / p.block_size + 1) * p.block_size) : n);
      // Page table entries of this wave's tiles: lane j of ids holds page j & 3 of
      // its tile 16 c + (j >> 2), ahead[0] those of the 16 tiles after, ahead[1] of
      // the next 16.  The pages' scales are gathered likewise, 16 tiles ahead.
      auto entries = [&](int i) {
        return page_entry(p, u.b, (static_cast<int64_t>(ta) + wave + static_cast<int64_t>(kStreamWaves) * (i + (lane >> 2))) * 4 + (lane & 3));
      };
      int ids = entries(0), ahead[2] = {entries(16), entries(32)};
      QRow<D> q_row;
      q_row.load(wanted ? p.q + ((row0 + wi) * p.num_q_heads + u.g * p.group + r % p.group) * D : nullptr);
      auto head_of = [&](int entry) { return static_cast<int64_t>(clamp_page(p, entry)) * p.num_kv_heads + u.g; };
      uint4 kx[2][NB], vx[2][NB];         // tile: [32-key block][chunk of the lane's key], [block][32-dim block]
      auto page_head = [&](int i, int j) { return head_of(__builtin_amdgcn_readlane(ids, (i & 15) * 4 + j)); };
      auto load_k = [&](int i, int blk) {
        const int64_t a = page_head(i, 2 * blk), b = page_head(i, 2 * blk + 1);
        const uint8_t *at = p.k_pages + (kpage ? b : a) * (kPageSize * D) + k_src;
#pragma unroll
        for (int j = 0; j < NB; ++j) kx[blk][j] = *reinterpret_cast<const uint4 *>(at + (j >> 1) * 64 + (j & 1) * 16);
      };
      auto load_v = [&](int i, int blk) {
        const int64_t a = page_head(i, 2 * blk), b = page_head(i, 2 * blk + 1);
        const uint8_t *at = p.v_pages + (h ? b : a) * (kPageSize * D) + col * kPageSize;
#pragma unroll
        for (int j = 0; j < NB; ++j) vx[blk][j] = *reinterpret_cast<const uint4 *>(at + j * 32 * kPageSize);
      };
      const int mine = (tb - ta - wave + kStreamWaves - 1) / kStreamWaves;       // tiles of this wave
#pragma unroll
      for (int blk = 0; blk < 2; ++blk) {
        load_k(0, blk);
        load_v(0, blk);
      }
      float ks = p.k_scales[head_of(ids)], vs = p.v_scales[head_of(ids)];
      float ks_next = p.k_scales[head_of(ahead[0])], vs_next = p.v_scales[head_of(ahead[0])];
      // factor of the scores, V's scale of the lane's page of block blk of the wave's tile i
      auto scale_of = [&](float x, int i, int blk) {
        const int at = (i & 15) * 4 + 2 * blk;
        const float a = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), at));
        const float b = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), at + 1));
        return h ? b : a;
      };
      i32x8 qh[NS], ql[NS];
      const float cq = make_q<D>(q_row, qh, ql) * p.scale_log2;

      f32x16 acc[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) acc[i] = f32x16{};
      float m = kNegHuge, l = 0.f;

      for (int i = 0; i < mine; ++i) {
        const int tile = ta + wave + kStreamWaves * i;
        // the next tile's entries (behind the last tile: that tile once more, from the cache)
        const int nx = min(i + 1, mine - 1);
        if ((i & 15) == 0 && i > 0) {
          ks = ks_next;
          vs = vs_next;
          ks_next = p.k_scales[head_of(ahead[0])];
          vs_next = p.v_scales[head_of(ahead[0])];
        }
        if ((nx & 15) == 0 && nx > i) {
          ids = ahead[0];
          ahead[0] = ahead[1];
          ahead[1] = entries(nx + 32);
        }
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          f32x16 s = f32x16{};
#pragma unroll
          for (int st = 0; st < NS; ++st) {
            const i32x8 k = operand(kx[blk][2 * st], kx[blk][2 * st + 1]);
            s = mfma_qk<FMT>(k, qh[st], s);
            s = mfma_qk<FMT>(k, ql[st], s);
          }
          const float c = k_factor(scale_of(ks, i, blk), cq), v = v_factor(scale_of(vs, i, blk));
          load_k(nx, blk);
          if (tile * kTile + kTile > u.p) {           // not every row sees every key
            const int key0 = tile * kTile + 32 * blk + 16 * h;
#pragma unroll
            for (int j = 0; j < 16; ++j) s[j] = j < seen - key0 ? s[j] : -__builtin_inff();
#pragma unroll
            for (int j = 0; j < NB; ++j) vx[blk][j] = zero_behind(vx[blk][j], n - key0);
          }
          bf16x8 pb[2];
          softmax_block<NB>(s, c, __builtin_amdgcn_logf(v), __builtin_amdgcn_rcpf(v), m, l, acc, pb);
#pragma unroll
          for (int j2 = 0; j2 < 2; ++j2)
#pragma unroll
            for (int j = 0; j < NB; ++j) {
              const uint4 d = vx[blk][j];
              acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(j2 ? widen8<FMT>(d.z, d.w) : widen8<FMT>(d.x, d.y), pb[j2], acc[j], 0, 0, 0);
            }
          load_v(nx, blk);
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
      const bool cut = ta > 0 || tb < u.tiles;
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
        const int64_t slot = deal.slot();
        float *dst = p.part_o + (slot * kStreamRows + jr) * D + part * (D / 8);
#pragma unroll
        for (int q = 0; q < D / 32; ++q) *reinterpret_cast<f32x4 *>(dst + 4 * q) = o[q];
        if (part == 0) {
          p.part_ml[(slot * kStreamRows + jr) * 2] = mm;
          p.part_ml[(slot * kStreamRows + jr) * 2 + 1] = ll;
        }
      } else if (row_wanted(p, u.b, u.w, u.row0, jrow)) {
        uint16_t *dst = p.out + ((row0 + jrow / p.group) * p.num_q_heads + u.g * p.group + jrow % p.group) * D + part * (D / 8);
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
          const uint2 w = {pack2(o[q][0], o[q][1]), pack2(o[q][2], o[q][3])};
          *reinterpret_cast<uint2 *>(dst + 4 * q) = w;
        }
      }
      __syncthreads();
    }
  } while (deal.next(u));
}

// ------------------------------------------------------- wide kernel
// Units of 64 * RG rows, RG = 1 or 2: four waves of 64 rows each, one on a SIMD,
// RG of them side by side on the rows and the others on further key tiles
// in turn.  Nothing goes through LDS but the final join of the tiles' groups: each
// wave loads K and V straight into operand registers, as the streaming kernel
// does, uses them for both of its 32-row blocks, and waves on the same tile share
// the loads through the CU's cache.
//
// A wave works on three (32-key block, row block) pairs at once: while the vector
// unit turns one's scores into probabilities, the matrix unit multiplies the next
// one's scores and adds P.V of the one before, all independent, instruction by
// instruction in turn.  Blocks of 32 rows of 4 heads each (RG = 2) behind 8 x 16384
// keys: 59 us with the join, 580 TFLOP/s; a tile takes 0.88 us.  Bound by what one
// wave can issue: a vector instruction every 6 clocks where two waves of a SIMD
// have one every 4, and a quarter of them move Q's operands, which the unified file
// holds beyond its first 256 registers.  (The same units on waves of 32 rows over
// tiles staged in LDS: 98 us where this form's first build took 74.)
template <int D, int FMT, int RG>
__global__ __launch_bounds__(256, 1) void attn_q8_wide_kernel(AttnQ8Params p) {
  constexpr int kRows = 64 * RG, KG = 4 / RG;
  constexpr int NB = D / 32, NS = D / 64;
  __shared__ __align__(16) float o_lds[KG > 1 ? (KG - 1) * RG : 1][KG > 1 ? 64 : 1][D + 4];
  __shared__ float ml_lds[4][64][2];
  if (p.gate && *p.gate == 0) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rg = wave % RG, kg = wave / RG;
  const int col = lane & 31, h = lane >> 5;
  const int kpage = (col >> 2) & 1;                   // the lane's key (K operand): its page of the block,
  const int k_src = (4 * (col >> 3) + (col & 3)) * D + h * 32;     // and byte in the page

  Deal<kRows> deal{p};
  Piece u;
  const bool work = deal.start(u);
  leave_note(p, deal, u, work);
  if (!work) return;
  do {
    const int ta = u.ta, tb = u.tb;
    const int n = u.p + u.w;
    int seen[2];
    bool wanted[2];
    int64_t q_at[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int r = u.qt * kRows + rg * 64 + b * 32 + col, wi = r / p.group;
      wanted[b] = row_wanted(p, u.b, u.w, u.row0, r);
      seen[b] = !wanted[b] ? 0 : (p.causal ? min(n, u.p + (wi / p.block_size + 1) * p.block_size) : n);
      q_at[b] = ((static_cast<int64_t>(u.row0) + wi) * p.num_q_heads + u.g * p.group + r % p.group) * D;
    }
    const bool busy = __builtin_amdgcn_ballot_w64(wanted[0] || wanted[1]) != 0;
    // (groups on other keys have the same rows: all or none of them are busy)
    float m[2] = {kNegHuge, kNegHuge}, l[2] = {0.f, 0.f};
    f32x16 acc[2][NB];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < NB; ++i) acc[b][i] = f32x16{};
    if (busy) {
      // page table entries and scales, as in the streaming kernel
      auto entries = [&](int i) {
        return page_entry(p, u.b, (static_cast<int64_t>(ta) + kg + static_cast<int64_t>(KG) * (i + (lane >> 2))) * 4 + (lane & 3));
      };
      int ids = entries(0), ahead[2] = {entries(16), entries(32)};
      QRow<D> q_row[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) q_row[b].load(wanted[b] ? p.q + q_at[b] : nullptr);
      auto head_of = [&](int entry) { return static_cast<int64_t>(clamp_page(p, entry)) * p.num_kv_heads + u.g; };
      uint4 kx[2][NB], vx[2][NB];
      auto page_head = [&](int i, int j) { return head_of(__builtin_amdgcn_readlane(ids, (i & 15) * 4 + j)); };
      auto load_k = [&](int i, int blk) {
        const int64_t a = page_head(i, 2 * blk), b = page_head(i, 2 * blk + 1);
        const uint8_t *at = p.k_pages + (kpage ? b : a) * (kPageSize * D) + k_src;
#pragma unroll
        for (int j = 0; j < NB; ++j) kx[blk][j] = *reinterpret_cast<const uint4 *>(at + (j >> 1) * 64 + (j & 1) * 16);
      };
      auto load_v = [&](int i, int blk) {
        const int64_t a = page_head(i, 2 * blk), b = page_head(i, 2 * blk + 1);
        const uint8_t *at = p.v_pages + (h ? b : a) * (kPageSize * D) + col * kPageSize;
#pragma unroll
        for (int j = 0; j < NB; ++j) vx[blk][j] = *reinterpret_cast<const uint4 *>(at + j * 32 * kPageSize);
      };
      const int mine = (tb - ta - kg + KG - 1) / KG;       // tiles of this wave
#pragma unroll
      for (int blk = 0; blk < 2; ++blk) {
        load_k(0, blk);
        load_v(0, blk);
      }
      float ks = p.k_scales[head_of(ids)], vs = p.v_scales[head_of(ids)];
      float ks_next = p.k_scales[head_of(ahead[0])], vs_next = p.v_scales[head_of(ahead[0])];
      auto scale_of = [&](float x, int i, int blk) {
        const int at = (i & 15) * 4 + 2 * blk;
        const float a = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), at));
        const float b = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), at + 1));
        return h ? b : a;
      };
      i32x8 qh[2][NS], ql[2][NS];
      float cq[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) cq[b] = make_q<D>(q_row[b], qh[b], ql[b]) * p.scale_log2;

      f32x16 s0, s1;
      bf16x8 p0[2], p1[2], wv[2][NB];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        p1[j] = bf16x8{};
#pragma unroll
        for (int i = 0; i < NB; ++i) wv[j][i] = bf16x8{};
      }
      // One step: probabilities of block blk, rows b, from s; into sn the scores of
      // block kblk, rows kb; P.V of pp with the V operands wv (widened here from
      // block vblk when `fresh`), rows pb.
      auto step = [&](auto widens, const uint4 (&fresh_v)[NB], f32x16 &s, int b, f32x16 &sn, const uint4 (&k)[NB], int kb,
                      const bf16x8 (&pp)[2], int pb, bf16x8 (&pc)[2], float ksc, float lv, float iv) {
        constexpr bool fresh = decltype(widens)::value;
        const float c = k_factor(ksc, cq[b]);
        float off = lv - m[b], t[2] = {0.f, 0.f}, e[16];
        auto value = [&](int i) {
          e[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, off));
          t[i & 1] += e[i];
          if (i & 1) {
            uint4 x = __builtin_bit_cast(uint4, pc[i >> 3]);
            reinterpret_cast<uint32_t *>(&x)[(i >> 1) & 3] = pack2(e[i - 1], e[i]);
            pc[i >> 3] = __builtin_bit_cast(bf16x8, x);
          }
        };
        constexpr int kQ = 2 * NS, kP = 2 * NB;
        __builtin_amdgcn_sched_barrier(0);
        sn = f32x16{};
#pragma unroll
        for (int i = 0; i < kQ; ++i) {
          sn = mfma_qk<FMT>(operand(k[i & ~1], k[i | 1]), i & 1 ? ql[kb][i >> 1] : qh[kb][i >> 1], sn);
#pragma unroll
          for (int j = 8 * i / kQ; j < 8 * (i + 1) / kQ; ++j) value(j);
          if (fresh && i == kQ - 1) wv[0][0] = widen8<FMT>(fresh_v[0].x, fresh_v[0].y);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < kP; ++i) {
          acc[pb][i % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wv[i / NB][i % NB], pp[i / NB], acc[pb][i % NB], 0, 0, 0);
          if (fresh && i + 1 < kP) {
            const uint4 d = fresh_v[(i + 1) % NB];
            wv[(i + 1) / NB][(i + 1) % NB] = (i + 1) / NB ? widen8<FMT>(d.z, d.w) : widen8<FMT>(d.x, d.y);
          }
#pragma unroll
          for (int j = 8 + 8 * i / kP; j < 8 + 8 * (i + 1) / kP; ++j) value(j);
          __builtin_amdgcn_sched_barrier(0);
        }
        float sum = (t[0] + t[1]) * iv;
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= kSumLimit)) != 0, 0)) {
          raise_reference<NB>(s, c, m[b], l[b], acc[b]);
          off = lv - m[b];
          t[0] = t[1] = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) value(i);
          sum = (t[0] + t[1]) * iv;
        }
        l[b] += sum;
      };
      auto mask = [&](f32x16 &s, int b, int key) {
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = j < seen[b] - key ? s[j] : -__builtin_inff();
      };

      s0 = f32x16{};
#pragma unroll
      for (int i = 0; i < 2 * NS; ++i)
        s0 = mfma_qk<FMT>(operand(kx[0][i & ~1], kx[0][i | 1]), i & 1 ? ql[0][i >> 1] : qh[0][i >> 1], s0);
      for (int i = 0; i < mine; ++i) {
        const int tile = ta + kg + KG * i;
        // the next tile's entries (behind the last tile: that tile once more, from the cache)
        const int nx = min(i + 1, mine - 1);
        if ((i & 15) == 0 && i > 0) {
          ks = ks_next;
          vs = vs_next;
          ks_next = p.k_scales[head_of(ahead[0])];
          vs_next = p.v_scales[head_of(ahead[0])];
        }
        if ((nx & 15) == 0 && nx > i) {
          ids = ahead[0];
          ahead[0] = ahead[1];
          ahead[1] = entries(nx + 32);
        }
        const bool masked = tile * kTile + kTile > u.p;
        const int key = tile * kTile + 16 * h;
        float v = v_factor(scale_of(vs, i, 0)), k = scale_of(ks, i, 0);
        float lv = __builtin_amdgcn_logf(v), iv = __builtin_amdgcn_rcpf(v);
        if (masked) mask(s0, 0, key);
        step(std::false_type{}, vx[0], s0, 0, s1, kx[0], 1, p1, 1, p0, k, lv, iv);
        load_k(nx, 0);
        if (masked) {
          mask(s1, 1, key);
#pragma unroll
          for (int j = 0; j < NB; ++j) vx[0][j] = zero_behind(vx[0][j], n - key);
        }
        step(std::true_type{}, vx[0], s1, 1, s0, kx[1], 0, p0, 0, p1, k, lv, iv);
        load_v(nx, 0);
        v = v_factor(scale_of(vs, i, 1)), k = scale_of(ks, i, 1);
        lv = __builtin_amdgcn_logf(v), iv = __builtin_amdgcn_rcpf(v);
        if (masked) mask(s0, 0, key + 32);
        step(std::false_type{}, vx[1], s0, 0, s1, kx[1], 1, p1, 1, p0, k, lv, iv);
        load_k(nx, 1);
        if (masked) {
          mask(s1, 1, key + 32);
#pragma unroll
          for (int j = 0; j < NB; ++j) vx[1][j] = zero_behind(vx[1][j], n - (key + 32));
        }
        step(std::true_type{}, vx[1], s1, 1, s0, kx[0], 0, p0, 0, p1, k, lv, iv);
        load_v(nx, 1);
      }
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i)
        acc[1][i % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wv[i / NB][i % NB], p1[i / NB], acc[1][i % NB], 0, 0, 0);
      l[0] = across_halves_add(l[0]);
      l[1] = across_halves_add(l[1]);
    }
    if constexpr (KG > 1) {
      if (kg > 0 && busy) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          if (h == 0) {
            ml_lds[wave][b * 32 + col][0] = m[b];
            ml_lds[wave][b * 32 + col][1] = l[b];
          }
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int a = 0; a < 4; ++a)
              *reinterpret_cast<f32x4 *>(&o_lds[wave - RG][b * 32 + col][j * 32 + 8 * a + 4 * h]) =
                  f32x4{acc[b][j][4 * a], acc[b][j][4 * a + 1], acc[b][j][4 * a + 2], acc[b][j][4 * a + 3]};
        }
      }
      __syncthreads();
      if (kg == 0 && busy) {
#pragma unroll
        for (int o = 1; o < KG; ++o)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int w = o * RG + rg;
            const float m2 = ml_lds[w][b * 32 + col][0], l2 = ml_lds[w][b * 32 + col][1];
            const float mn = fmaxf(m[b], m2);
            const float wa = __builtin_amdgcn_exp2f(m[b] - mn), wb = __builtin_amdgcn_exp2f(m2 - mn);
            m[b] = mn;
            l[b] = l[b] * wa + l2 * wb;
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
              for (int a = 0; a < 4; ++a) {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(&o_lds[w - RG][b * 32 + col][j * 32 + 8 * a + 4 * h]);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[b][j][4 * a + i] = acc[b][j][4 * a + i] * wa + x[i] * wb;
              }
          }
      }
      __syncthreads();
    }
    if (kg == 0 && busy) {
      const bool cut = ta > 0 || tb < u.tiles;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if (cut) {
          const int64_t at = deal.slot() * kRows + rg * 64 + b * 32 + col;
          if (h == 0) {
            p.part_ml[at * 2] = m[b];
            p.part_ml[at * 2 + 1] = l[b];
          }
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int a = 0; a < 4; ++a)
              *reinterpret_cast<f32x4 *>(p.part_o + at * D + j * 32 + 8 * a + 4 * h) =
                  f32x4{acc[b][j][4 * a], acc[b][j][4 * a + 1], acc[b][j][4 * a + 2], acc[b][j][4 * a + 3]};
        } else if (wanted[b]) {
          const float inv = 1.f / l[b];
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int a = 0; a < 4; ++a)
              *reinterpret_cast<uint2 *>(p.out + q_at[b] + j * 32 + 8 * a + 4 * h) =
                  uint2{pack2(acc[b][j][4 * a] * inv, acc[b][j][4 * a + 1] * inv),
                        pack2(acc[b][j][4 * a + 2] * inv, acc[b][j][4 * a + 3] * inv)};
        }
      }
    }
  } while (deal.next(u));
}

// ------------------------------------------------------- tile kernel
// Units of 256 rows: a workgroup of eight waves of 32 rows, two on a SIMD, stages
// every key tile once in LDS for all of them.
//
// K goes into LDS as it is (half the bytes bf16 would take), V as bf16, converted
// once per workgroup on the way: two planes of 8 keys by dim, 16 bytes each, as
// P.V's operand reads them.  Rows of K lie in the order of the operand's rows,
// their 16-byte chunks XOR-swizzled so that any eight rows' equal chunks fall on
// different banks.
//
// A wave works on three 32-key blocks at once, as in the wide kernel.  So
// iteration t reads K of tiles t and t + 1 and V of t - 1 and t, from three LDS
// buffers each; it writes K of t + 2 and V of t + 1 from registers, and loads K of
// t + 4 and V of t + 3 into them: one barrier a tile, two tiles' time for a load.
//
// Windows of 128 rows of 4 heads behind 64 x 4096 to 32768 keys: 1.19 ms, 1.05
// PFLOP/s, where a large bf16 product reaches 1.23 on this card.  A tile takes 1.46
// us on one CU alone and 2.1 with all of them at work: bound by the matrix and
// vector units at the clock that the board's power leaves (about 2.0 GHz).
constexpr int kTileRows = 256, kTileThreads = 512;

template <int D, int FMT>
__global__ __launch_bounds__(kTileThreads, 1) void attn_q8_tile_kernel(AttnQ8Params p) {
  constexpr int NB = D / 32, NS = D / 64;
  constexpr int kChunks = D / 16;         // 16-byte chunks of a K row
  constexpr int kStagers = 4 * D;         // threads that stage a tile: 16 bytes of K and of V each
  constexpr int kK = kTile * D, kV = kTile * D * 2;      // bytes of a tile in LDS
  constexpr int kBuf = kK + kV;
  __shared__ __align__(16) uint8_t lds[3 * kBuf];
  __shared__ __align__(16) float sc[3][4][4];            // per page: K scale, log2 and reciprocal of V's
  if (p.gate && *p.gate == 0) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, h = lane >> 5;

  Deal<kTileRows> deal{p};
  Piece u;
  const bool work = deal.start(u);
  leave_note(p, deal, u, work);
  if (!work) return;
  // staging: this thread's 16 bytes of page spage: of K a slot's chunk, of V a dim.
  // (D = 64: two threads do the same; a branch around the loads would leave the
  // compiler unsure of how many are in flight, and it would wait for all)
  const int spage = __builtin_amdgcn_readfirstlane((tid % kStagers) / D), sdim = tid % D;
  const bool scaler = wave % (D / 64) == 0;              // the wave with dim 0 stages the page's scales
  const int kslot = sdim / kChunks;
  const int krow = 32 * (spage >> 1) + 8 * (kslot >> 2) + 4 * (spage & 1) + (kslot & 3);
  const int k_dst = krow * D + (((sdim % kChunks) ^ (D == 128 ? krow & 7 : (krow >> 1) & 3)) * 16);
  const int v_dst = kK + (spage * 2 * D + sdim) * 16;
  // operand reads: 16-byte chunks of the lane's K row (block 0), of its V rows
  int k_at[2 * NS];
#pragma unroll
  for (int i = 0; i < 2 * NS; ++i)
    k_at[i] = col * D + (((4 * (i >> 1) + 2 * h + (i & 1)) ^ (D == 128 ? col & 7 : (col >> 1) & 3)) * 16);
  const int v_at = kK + (h * 2 * D + col) * 16;

  do {
    const int ta = u.ta, tb = u.tb;
    const int n = u.p + u.w;
    const int r = u.qt * kTileRows + wave * 32 + col;
    const bool wanted = row_wanted(p, u.b, u.w, u.row0, r);
    const bool mine = __builtin_amdgcn_ballot_w64(wanted) != 0;
    if (!p.block_flags || __syncthreads_or(mine)) {
      const int wi = r / p.group;
      const int seen = !wanted ? 0 : (p.causal ? min(n, u.p + (wi / p.block_size + 1) * p.block_size) : n);
      const int64_t q_at = ((static_cast<int64_t>(u.row0) + wi) * p.num_q_heads + u.g * p.group + r % p.group) * D;
      const int iters = tb - ta;
      // Page table entries of this wave's page: lane j of ids holds that of tile
      // 64 c + j, ahead those of the 64 after.
      auto entries = [&](int it0) { return page_entry(p, u.b, (static_cast<int64_t>(ta) + it0 + lane) * 4 + spage); };
      int ids = entries(0), ahead = entries(64);
      QRow<D> q_row;
      q_row.load(wanted ? p.q + q_at : nullptr);
      // (page, head) row of the pools for tile it, asked for in order
      auto page_head = [&](int it) {
        return static_cast<int64_t>(clamp_page(p, __builtin_amdgcn_readlane(ids, it & 63))) * p.num_kv_heads + u.g;
      };
      struct KRegs {
        uint4 k;
        float ks, vs;
      };
      auto load_k = [&](KRegs &x, int64_t ph) {
        x.k = *reinterpret_cast<const uint4 *>(p.k_pages + ph * (kPageSize * D) + sdim * 16);
        x.ks = p.k_scales[ph];
        x.vs = p.v_scales[ph];
      };
      auto load_v = [&](uint4 &x, int64_t ph) {
        x = *reinterpret_cast<const uint4 *>(p.v_pages + ph * (kPageSize * D) + sdim * 16);
      };
      auto stage_k = [&](const KRegs &x, uint8_t *buf, int sbuf) {
        *reinterpret_cast<uint4 *>(buf + k_dst) = x.k;
        if (scaler) {
          const float vs = v_factor(x.vs);
          const f32x4 w = {x.ks, __builtin_amdgcn_logf(vs), __builtin_amdgcn_rcpf(vs), 0.f};
          if (sdim == 0) *reinterpret_cast<f32x4 *>(sc[sbuf][spage]) = w;
        }
      };
      auto stage_v = [&](uint4 x, uint8_t *buf, int it) {
        const int key = (ta + it) * kTile;
        if (key + kTile > n) x = zero_behind(x, n - (key + spage * 16));
        bf16x8 *at = reinterpret_cast<bf16x8 *>(buf + v_dst);
        at[0] = widen8<FMT>(x.x, x.y);
        at[D] = widen8<FMT>(x.z, x.w);
      };

      // tiles 0 and 1 of K, 0 of V in LDS; tiles 2 and 3 of K, 1 and 2 of V on their way
      KRegs ka, kb;
      uint4 va, vb;
      const int64_t ph0 = page_head(0), ph1 = page_head(1), ph2 = page_head(2);
      int64_t ph = page_head(3);
      load_k(ka, ph0);
      load_v(va, ph0);
      load_k(kb, ph1);
      load_v(vb, ph1);
      i32x8 qh[NS], ql[NS];
      const float cq = make_q<D>(q_row, qh, ql) * p.scale_log2;
      stage_k(ka, lds, 0);
      load_k(ka, ph2);
      stage_v(va, lds, 0);
      va = vb;
      load_v(vb, ph2);
      stage_k(kb, lds + kBuf, 1);
      load_k(kb, ph);

      f32x16 acc[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) acc[i] = f32x16{};
      float m = kNegHuge, l = 0.f;
      f32x16 s0, s1;
      bf16x8 p0[2], p1[2];
      p1[0] = p1[1] = bf16x8{};
      // Operands of the next scores and the page factors of the next block: read from
      // LDS while the block before is worked on.
      uint4 ko[2 * NS];
      f32x4 w;
      auto read_k = [&](const uint8_t *buf, int blk, int i) { ko[i] = *reinterpret_cast<const uint4 *>(buf + k_at[i] + blk * 32 * D); };
      auto read_w = [&](int buf, int blk) { w = *reinterpret_cast<const f32x4 *>(&sc[buf][2 * blk + h][0]); };
      // probabilities of a 32-key block from its scores s; the scores sn of the next
      // block (from ko) and P.V of the one before (pp, vbuf, vblk) beside them
      auto block = [&](f32x16 &s, f32x16 &sn, const bf16x8 (&pp)[2], const uint8_t *vbuf, int vblk, bf16x8 (&pc)[2], int key0,
                       bool masked, const uint8_t *kbuf, int kblk, int wbuf, int wblk) {
        if (masked) {
          const int left = seen - (key0 + 16 * h);
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = i < left ? s[i] : -__builtin_inff();
        }
        bf16x8 vo[2 * NB];
        const bf16x8 *vp = reinterpret_cast<const bf16x8 *>(vbuf + v_at) + vblk * 4 * D;
        const float c = k_factor(w[0], cq), lv = w[1], iv = w[2];
        float off = lv - m, sum, e[16], t[2] = {0.f, 0.f};
        auto value = [&](int i) {
          e[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, off));
          t[i & 1] += e[i];
          if (i & 1) {
            uint4 x = __builtin_bit_cast(uint4, pc[i >> 3]);
            reinterpret_cast<uint32_t *>(&x)[(i >> 1) & 3] = pack2(e[i - 1], e[i]);
            pc[i >> 3] = __builtin_bit_cast(bf16x8, x);
          }
        };
        // the vector unit's work, and the reads, between the matrix unit's
        constexpr int kQ = 2 * NS, kP = 2 * NB;
        __builtin_amdgcn_sched_barrier(0);
        sn = f32x16{};
#pragma unroll
        for (int i = 0; i < kQ; ++i) {
#pragma unroll
          for (int j = i * NB / NS; j < (i + 1) * NB / NS; ++j) vo[j] = vp[(j / NB) * D + (j % NB) * 32];
          sn = mfma_qk<FMT>(operand(ko[i & ~1], ko[i | 1]), i & 1 ? ql[i >> 1] : qh[i >> 1], sn);
#pragma unroll
          for (int j = 8 * i / kQ; j < 8 * (i + 1) / kQ; ++j) value(j);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < kP; ++i) {
          if (i >= kP / 2) {
            if (i == kP / 2) read_w(wbuf, wblk);
            read_k(kbuf, kblk, i - kP / 2);
          }
          acc[i % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vo[i], pp[i / NB], acc[i % NB], 0, 0, 0);
#pragma unroll
          for (int j = 8 + 8 * i / kP; j < 8 + 8 * (i + 1) / kP; ++j) value(j);
          __builtin_amdgcn_sched_barrier(0);
        }
        sum = (t[0] + t[1]) * iv;
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= kSumLimit)) != 0, 0)) {
          raise_reference<NB>(s, c, m, l, acc);
          off = lv - m;
          t[0] = t[1] = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) value(i);
          sum = (t[0] + t[1]) * iv;
        }
        l += sum;
      };

      __syncthreads();
      if (mine) {
        s0 = f32x16{};
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const i32x8 k = operand(*reinterpret_cast<const uint4 *>(lds + k_at[2 * i]), *reinterpret_cast<const uint4 *>(lds + k_at[2 * i + 1]));
          s0 = mfma_qk<FMT>(k, qh[i], s0);
          s0 = mfma_qk<FMT>(k, ql[i], s0);
        }
#pragma unroll
        for (int i = 0; i < 2 * NS; ++i) read_k(lds, 1, i);
        read_w(0, 0);
      }
      // buffers of tiles it, it + 1, it + 2, and of it - 1 (the first P.V adds zeros: any V in place will do)
      uint8_t *b0 = lds, *b1 = lds + kBuf, *b2 = lds + 2 * kBuf, *prev = lds;
      int i0 = 0, i1 = 1, i2 = 2;
      auto iteration = [&](int it, KRegs &kr, uint4 &vr) {
        const int key = (ta + it) * kTile;
        const bool masked = key + kTile > u.p;
        if (mine) block(s0, s1, p1, prev, 1, p0, key, masked, b1, 0, i0, 1);
        stage_v(vr, b1, it + 1);
        load_v(vr, ph);                     // tile it + 3
        if (mine) block(s1, s0, p0, b0, 0, p1, key + 32, masked, b1, 1, i1, 0);
        stage_k(kr, b2, i2);
        if (((it + 4) & 63) == 0) {
          ids = ahead;
          ahead = entries(it + 4 + 64);
        }
        ph = page_head(it + 4);
        __syncthreads();
        load_k(kr, ph);                     // tile it + 4
        prev = b0;
        b0 = b1;
        b1 = b2;
        b2 = prev;
        const int i = i0;
        i0 = i1;
        i1 = i2;
        i2 = i;
      };
      int it = 0;
      for (; it + 1 < iters; it += 2) {
        iteration(it, ka, va);
        iteration(it + 1, kb, vb);
      }
      if (it < iters) iteration(it, ka, va);
      if (mine) {
        const bf16x8 *vp = reinterpret_cast<const bf16x8 *>(prev + v_at) + 4 * D;
#pragma unroll
        for (int i = 0; i < 2 * NB; ++i)
          acc[i % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vp[(i / NB) * D + (i % NB) * 32], p1[i / NB], acc[i % NB], 0, 0, 0);
      }
      l = across_halves_add(l);
      if (ta > 0 || tb < u.tiles) {
        const int64_t at = deal.slot() * kTileRows + wave * 32 + col;
        if (h == 0) {
          p.part_ml[at * 2] = m;
          p.part_ml[at * 2 + 1] = l;
        }
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int a = 0; a < 4; ++a)
            *reinterpret_cast<f32x4 *>(p.part_o + at * D + j * 32 + 8 * a + 4 * h) =
                f32x4{acc[j][4 * a], acc[j][4 * a + 1], acc[j][4 * a + 2], acc[j][4 * a + 3]};
      } else if (wanted) {
        const float inv = 1.f / l;
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int a = 0; a < 4; ++a)
            *reinterpret_cast<uint2 *>(p.out + q_at + j * 32 + 8 * a + 4 * h) =
                uint2{pack2(acc[j][4 * a] * inv, acc[j][4 * a + 1] * inv), pack2(acc[j][4 * a + 2] * inv, acc[j][4 * a + 3] * inv)};
      }
      __syncthreads();
    }
  } while (deal.next(u));
}

// ------------------------------------------------------------- the join
// Workgroup x joins the unit that the note of share x + 1 names, if it names one.
// A block takes RPB rows of it; a row's dims lie across D / 4 lanes, and its parts
// are dealt to G groups of lanes, whose results meet in LDS.  Bound by the parts'
// bytes where units are large (4 D per row and part: 67 MB in 11 us), by the chain
// note -> statistics -> accumulators otherwise (4 us).
template <int D, int ROWS, int RPB>
__global__ __launch_bounds__(256) void attn_q8_join_kernel(AttnQ8Params p) {
  constexpr int kLanes = D / 4, G = 256 / (kLanes * RPB);
  __shared__ __align__(16) float o_lds[RPB][G][D];
  __shared__ float ml_lds[RPB][G][2];
  if (p.gate && *p.gate == 0) return;
  const int64_t wg = static_cast<int64_t>(blockIdx.x) + 1;
  const JoinNote n = *reinterpret_cast<const JoinNote *>(p.notes + 8 * wg);
  if (n.parts == 0) return;
  const int tid = threadIdx.x, lane = tid % kLanes, group = tid / kLanes % G, row = tid / (kLanes * G);
  const int r_in = static_cast<int>(blockIdx.y) * RPB + row, r = n.qt * ROWS + r_in;
  const bool wanted = row_wanted(p, n.b, n.w, n.row0, r);
  if (RPB == 1 ? !wanted : !__syncthreads_or(wanted)) return;
  float m = kNegHuge, l = 0.f;
  f32x4 o = {};
  constexpr int U = 4;                              // parts in flight
  for (int i0 = group; i0 < n.parts; i0 += G * U) {
    float pm[U], pl[U];
    f32x4 v[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int i = min(i0 + k * G, n.parts - 1);
      const int64_t at = (i == 0 ? n.slot : 2 * (wg + i - 1)) * ROWS + r_in;
      pm[k] = p.part_ml[at * 2];
      pl[k] = p.part_ml[at * 2 + 1];
      v[k] = *reinterpret_cast<const f32x4 *>(p.part_o + at * D + lane * 4);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (i0 + k * G >= n.parts) continue;
      const float mn = fmaxf(m, pm[k]);
      const float a = __builtin_amdgcn_exp2f(m - mn), b = __builtin_amdgcn_exp2f(pm[k] - mn);
      m = mn;
      l = l * a + pl[k] * b;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = o[j] * a + v[k][j] * b;
    }
  }
  if constexpr (G > 1) {
    *reinterpret_cast<f32x4 *>(&o_lds[row][group][lane * 4]) = o;
    if (lane == 0) {
      ml_lds[row][group][0] = m;
      ml_lds[row][group][1] = l;
    }
    __syncthreads();
    if (group != 0) return;
#pragma unroll
    for (int k = 1; k < G; ++k) {
      const float pm = ml_lds[row][k][0], pl = ml_lds[row][k][1];
      const f32x4 v = *reinterpret_cast<const f32x4 *>(&o_lds[row][k][lane * 4]);
      const float mn = fmaxf(m, pm);
      const float a = __builtin_amdgcn_exp2f(m - mn), b = __builtin_amdgcn_exp2f(pm - mn);
      m = mn;
      l = l * a + pl * b;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = o[j] * a + v[j] * b;
    }
  }
  if (!wanted) return;
  const float inv = 1.f / l;
  uint16_t *dst = p.out + ((static_cast<int64_t>(n.row0) + r / p.group) * p.num_q_heads + n.g * p.group + r % p.group) * D + lane * 4;
  *reinterpret_cast<uint2 *>(dst) = uint2{pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv)};
}

// Few rows can have many parts: two rows a block.  Many rows have few parts each.
template <int D, int ROWS>
void launch_join(const AttnQ8Params &p, hipStream_t stream) {
  constexpr int kRows = ROWS <= 32 ? 2 : 256 / (D / 4);
  const int rows = static_cast<int>(min(static_cast<int64_t>(ROWS), static_cast<int64_t>(p.group) * p.max_window));
  hipLaunchKernelGGL((attn_q8_join_kernel<D, ROWS, kRows>),
                     dim3(static_cast<unsigned>(p.wgs - 1), static_cast<unsigned>((rows + kRows - 1) / kRows)), dim3(256), 0,
                     stream, p);
}

template <int D, int FMT>
hipError_t launch(const AttnQ8Params &p, const AttnQ8Plan &plan, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(plan.wgs));
  const bool join = plan.split && plan.wgs > 1;
  hipError_t e;
  if (plan.rows == 32) {
    hipLaunchKernelGGL((attn_q8_stream_kernel<D, FMT>), grid, dim3(256), 0, stream, p);
    e = hipGetLastError();
    if (e == hipSuccess && join) launch_join<D, 32>(p, stream);
  } else if (plan.rows == 64) {
    hipLaunchKernelGGL((attn_q8_wide_kernel<D, FMT, 1>), grid, dim3(256), 0, stream, p);
    e = hipGetLastError();
    if (e == hipSuccess && join) launch_join<D, 64>(p, stream);
  } else if (plan.rows == 128) {
    hipLaunchKernelGGL((attn_q8_wide_kernel<D, FMT, 2>), grid, dim3(256), 0, stream, p);
    e = hipGetLastError();
    if (e == hipSuccess && join) launch_join<D, 128>(p, stream);
  } else {
    hipLaunchKernelGGL((attn_q8_tile_kernel<D, FMT>), grid, dim3(kTileThreads), 0, stream, p);
    e = hipGetLastError();
    if (e == hipSuccess && join) launch_join<D, 256>(p, stream);
  }
  return e == hipSuccess ? hipGetLastError() : e;
}

}  // namespace

hipError_t launch_attn_q8(const AttnQ8Params &p, const AttnQ8Plan &plan, int head_dim, int format, hipStream_t stream) {
  if (head_dim == 128)
    return format == MBE_Q8_E4M3 ? launch<128, MBE_Q8_E4M3>(p, plan, stream) : launch<128, MBE_Q8_E5M2>(p, plan, stream);
  return format == MBE_Q8_E4M3 ? launch<64, MBE_Q8_E4M3>(p, plan, stream) : launch<64, MBE_Q8_E5M2>(p, plan, stream);
}

}  // namespace mbe
