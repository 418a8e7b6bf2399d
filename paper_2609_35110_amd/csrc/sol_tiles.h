// Tiles of bf16 rows staged in LDS and the MFMA fragments read from them:
// shared by the linear (sol_lin_attn.hip) and differential
// (sol_diff_attn.hip) attention.
#pragma once

#include "sol_device.h"

namespace sol {
namespace {

// LDS row stride of a staged tile, elements: 288 bytes = 8 banks past a whole
// turn of the 64, so that the 16-byte reads along rows (8 rows at a time) and
// the transpose reads (4 rows of 32 bytes) both touch every bank once.
constexpr int kStride = D + 16;

// An MFMA 32 x 32 x 16 (bf16 in, fp32 out) takes A and B with lane l holding
// row (column) l % 32 and eight of the sixteen inner places, and leaves lane l
// column l % 32 of the result, register r its row 8 (r / 4) + 4 (l / 32) + r % 4.
// The inner places may come in any order that A and B share.  So a result
// rounded to bf16 is, register for register, the operand of a product over its
// rows, whose other operand column8 reads in that row order.
__device__ __forceinline__ f32x16 mfma(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// This lane's place in a transpose read (element offset into a tile).
__device__ __forceinline__ int column_offset(int lane) {
  const int g16 = lane >> 4, i16 = lane & 15;
  return (4 * (g16 >> 1) + (i16 >> 2)) * kStride + 16 * (g16 & 1) + 4 * (i16 & 3);
}
// Eight values of column lane % 32 (from p, which includes column_offset):
// rows {0..3, 8..11} + 4 (lane / 32), the order above.
__device__ __forceinline__ bf16x8 column8(const uint16_t* p) {
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 8 * kStride));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// Eight values of row lane % 32, places 16 kk + 8 (lane / 32) on.
__device__ __forceinline__ bf16x8 row8(const uint16_t* tile, int lane, int kk) {
  return *reinterpret_cast<const bf16x8*>(tile + (lane & 31) * kStride + 16 * kk + 8 * (lane >> 5));
}

// Eight consecutive registers of a result as the operand of the next product.
__device__ __forceinline__ bf16x8 operand8(const f32x16& s, int x) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = s[8 * x + i];
  return __builtin_bit_cast(bf16x8, pack_bf16x8(f));
}

// kRows rows on their way into LDS, moved by kThreads threads (thread t of them
// holds 16-byte chunk t % 16 of rows t / 16 + (kThreads / 16) u).  Rows from
// `rows` on are zero and not read.
template <int kRows, int kThreads>
struct Stage {
  static constexpr int kStep = kThreads / 16;
  uint4 x[kRows / kStep];
  __device__ __forceinline__ void load(const uint16_t* p, int64_t sn, int row0, int rows, int t) {
    const int r = t >> 4, cc = t & 15;
#pragma unroll
    for (int u = 0; u < kRows / kStep; ++u) {
      const int i = row0 + r + kStep * u;
      x[u] = make_uint4(0, 0, 0, 0);
      if (i < rows) x[u] = *reinterpret_cast<const uint4*>(p + (int64_t)i * sn + cc * 8);
    }
  }
  __device__ __forceinline__ void store(uint16_t* tile, int t) const {
    const int r = t >> 4, cc = t & 15;
#pragma unroll
    for (int u = 0; u < kRows / kStep; ++u) *reinterpret_cast<uint4*>(tile + (r + kStep * u) * kStride + cc * 8) = x[u];
  }
};

// The larger (sum) of the two lanes l and l ^ 32, in both.
__device__ __forceinline__ float both_max(float x) { return fmaxf(x, __shfl_xor(x, 32)); }
__device__ __forceinline__ float both_sum(float x) { return x + __shfl_xor(x, 32); }

}  // namespace
}  // namespace sol
