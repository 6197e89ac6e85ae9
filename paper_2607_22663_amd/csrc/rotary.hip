// Rotary positions of the queries and keys of ragged sequences, gfx950.
//
// A pair (x, y) at position n turns by a = 2 pi frac(n t), t its frequency in
// turns per position.  t is held in 64-bit fixed point, so n t modulo one turn
// is the low 64 bits of an integer product: the phase is exact at any
// position, where fp32 radians lose a whole radian at n = 2^24.  The sine and
// cosine instructions take turns, so the top 32 bits convert straight into
// their argument; arithmetic is fp32, rounded once to bf16.
//
// A thread owns 16 dims (8 pairs) of a row and HEADS heads of it: its sines and
// cosines are computed once and used for every one of its heads, and the loads of
// all its heads are in flight together.  Eight threads (D = 128) cover a head's
// row, 16 bytes a lane and access.  2 bytes in and 2 out a value: bound by HBM for
// long inputs (4.4 TB/s on 75000 rows of 20 heads), by latency for a window's rows.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "q8.h"
#include "q8_device.h"

namespace mbe {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ inline float bf_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ inline float bf_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ inline uint32_t pair(float lo, float hi) {
  bf16x2 r;
  r[0] = static_cast<__bf16>(lo);
  r[1] = static_cast<__bf16>(hi);
  return __builtin_bit_cast(uint32_t, r);
}

template <int D, int HEADS>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p) {
  constexpr int kChunks = D / 16;
  const int b = blockIdx.y;
  const int len = min(max(p.lens[b], 0), p.max_len);
  const int item = static_cast<int>(blockIdx.x) * 256 + static_cast<int>(threadIdx.x);
  if (static_cast<int>(blockIdx.x) * (256 / kChunks) >= len) return;
  const int t = item / kChunks, c = item % kChunks;
  const int64_t row = rows_before(p.lens, b, p.max_len) + t;
  if (t >= len || row >= p.total_rows) return;
  const int heads = p.num_q_heads + p.num_kv_heads;
  const int h0 = static_cast<int>(blockIdx.z) * HEADS;
  // The two 8-dim chunks of this thread: c-th of the rotated dims' halves (or of the
  // other dims' halves), so that neighbours' chunks lie next to each other.
  const int half = p.rot_dim / 2;
  const bool rotated = c * 16 < p.rot_dim;
  const int d0 = rotated ? c * 8 : half + c * 8, d1 = d0 + (rotated ? half : D / 2 - half);
  uint4 x[HEADS][2];
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int h = h0 + i;
    if (h >= heads) continue;
    const uint16_t *at = h < p.num_q_heads ? p.q + row * p.q_stride + static_cast<int64_t>(h) * D
                                           : p.k + row * p.k_stride + static_cast<int64_t>(h - p.num_q_heads) * D;
    x[i][0] = *reinterpret_cast<const uint4 *>(at + d0);
    x[i][1] = *reinterpret_cast<const uint4 *>(at + d1);
  }
  float cs[8], sn[8];
  if (rotated) {
    const uint32_t n = static_cast<uint32_t>(max(p.start_pos[b], 0)) + static_cast<uint32_t>(t);
    const float sign = p.inverse ? -p.scale : p.scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // pairs of the chunks: c * 8 + i, or four of each chunk
      const int pair_at = p.interleaved ? (i < 4 ? d0 : d1) / 2 + (i & 3) : c * 8 + i;
      const uint64_t turns = p.turns[pair_at] * n;
      const float a = static_cast<float>(static_cast<int32_t>(turns >> 32)) * 0x1p-32f;    // in [-1/2, 1/2]
      cs[i] = __builtin_amdgcn_cosf(a) * p.scale;
      sn[i] = __builtin_amdgcn_sinf(a) * sign;
    }
  }
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int h = h0 + i;
    if (h >= heads) continue;
    uint32_t *u = reinterpret_cast<uint32_t *>(x[i]);
    if (rotated && p.interleaved) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = bf_lo(u[j]), e = bf_hi(u[j]);
        u[j] = pair(a * cs[j] - e * sn[j], e * cs[j] + a * sn[j]);
      }
    } else if (rotated) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float a0 = bf_lo(u[j]), a1 = bf_hi(u[j]), e0 = bf_lo(u[j + 4]), e1 = bf_hi(u[j + 4]);
        u[j] = pair(a0 * cs[2 * j] - e0 * sn[2 * j], a1 * cs[2 * j + 1] - e1 * sn[2 * j + 1]);
        u[j + 4] = pair(e0 * cs[2 * j] + a0 * sn[2 * j], e1 * cs[2 * j + 1] + a1 * sn[2 * j + 1]);
      }
    }
    uint16_t *at = h < p.num_q_heads ? p.q_out + row * p.q_out_stride + static_cast<int64_t>(h) * D
                                     : p.k_out + row * p.k_out_stride + static_cast<int64_t>(h - p.num_q_heads) * D;
    *reinterpret_cast<uint4 *>(at + d0) = x[i][0];
    *reinterpret_cast<uint4 *>(at + d1) = x[i][1];
  }
}

template <int D, int HEADS>
void launch_heads(const RotaryParams &p, hipStream_t stream) {
  const int heads = p.num_q_heads + p.num_kv_heads;
  const int64_t items = static_cast<int64_t>(p.max_len) * (D / 16);
  const dim3 grid(static_cast<unsigned>((items + 255) / 256), static_cast<unsigned>(p.batch),
                  static_cast<unsigned>((heads + HEADS - 1) / HEADS));
  hipLaunchKernelGGL((rotary_kernel<D, HEADS>), grid, dim3(256), 0, stream, p);
}

// Two heads a thread spread few rows over the chip, ten spare the sines of many.
// us with 2 / 4 / 10 heads a thread, D = 128, 20 heads: 128 rows 4.2 / 4.8 / 7.2,
// 75000 rows 186 / 183 / 176.
template <int D>
hipError_t launch(const RotaryParams &p, hipStream_t stream) {
  const int64_t rows = static_cast<int64_t>(p.total_rows) * (p.num_q_heads + p.num_kv_heads);
  if (rows < 65536) launch_heads<D, 2>(p, stream);
  else launch_heads<D, 10>(p, stream);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryParams &p, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch<128>(p, stream) : launch<64>(p, stream);
}

}  // namespace mbe
