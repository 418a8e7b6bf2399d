// What the softmax attentions' kernels share (sol_diff_attn.hip,
// sol_cross_attn.hip): a wave's rows under the running maximum and sum, scores,
// exponentials, and rows on their way out.
#pragma once

#include "sol_tiles.h"

namespace sol {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;
// A maximum below every score; finite, so that differences with it are not NaN.
constexpr float kNoMax = -1e30f;
// Binades by which a row's scores may pass the maximum it is held to before it
// is raised: P has bf16's exponents, so only the fp32 sums' range matters.
constexpr float kSlack = 8.0f;

// The keys of split i of n: whole tiles, as even as they come.
__device__ __forceinline__ int2 split_keys(int klen, int i, int n, int tile) {
  const int tiles = (klen + tile - 1) / tile;
  const int per = (tiles + n - 1) / n;
  return make_int2(min(i * per * tile, klen), min((i + 1) * per * tile, klen));
}

// 32 rows of one map: a lane's row is lane % 32.
struct MapRows {
  f32x16 o[4];  // O^T: dims 32t + 8(r/4) + 4(lane/32) + r%4
  float m;      // maximum held to (raw scores)
  // Sums over this lane's half of the keys: of P as the product takes it, rounded,
  // which O is divided by (a row that one key has most of gets that key's value
  // whole, whatever its P's rounding), and of P before that for the log sum.
  float l, exact;
};
// sum + the two values of a word
__device__ __forceinline__ float add_bf16x2(uint32_t x, float sum) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), __builtin_bit_cast(bf16x2, 0x3f803f80u), sum, false);
}
__device__ __forceinline__ float add_bf16x8(const bf16x8& p, float sum) {
  const uint4 x = __builtin_bit_cast(uint4, p);
  return add_bf16x2(x.x, add_bf16x2(x.y, add_bf16x2(x.z, add_bf16x2(x.w, sum))));
}
__device__ __forceinline__ void clear(MapRows& x) {
#pragma unroll
  for (int t = 0; t < 4; ++t) x.o[t] = f32x16{};
  x.m = kNoMax;
  x.l = x.exact = 0.0f;
}

// The running maximum: raised, with the sums, when any row of the wave passes
// the one it is held to by more than kSlack binades.
template <int kBlocks>
__device__ __forceinline__ void raise_max(MapRows& x, const f32x16 (&s)[kBlocks], float c) {
  float top = s[0][0];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
  top = both_max(top);
  if (__any((top - x.m) * c > kSlack)) {
    const float m = fmaxf(x.m, top);
    const float keep = __builtin_amdgcn_exp2f((x.m - m) * c);
    x.l *= keep;
    x.exact *= keep;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) x.o[t][r] *= keep;
    x.m = m;
  }
}

// P of 32 keys in place of their scores, and its sum before any rounding.
__device__ __forceinline__ void exponentials(MapRows& x, f32x16& s, float c) {
  const float mc = x.m * c;
  float a = 0.0f, b = 0.0f;
#pragma unroll
  for (int r = 0; r < 16; r += 2) {
    s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -mc));
    s[r + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + 1], c, -mc));
    a += s[r];
    b += s[r + 1];
  }
  x.exact += a + b;
}

// Scores of 32 keys (rows of the result) for the wave's 32 rows.
__device__ __forceinline__ f32x16 scores(const uint16_t* tk, const bf16x8 (&qf)[8], int lane) {
  f32x16 s = {};
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) s = mfma(row8(tk, lane, kk), qf[kk], s);
  return s;
}

// Scores of keys past `last` (this lane's row) go: register r is key
// key0 + 8 (r/4) + r%4.
__device__ __forceinline__ void mask(f32x16& s, int key0, int last) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (key0 + 8 * (r >> 2) + (r & 3) > last) s[r] = -__builtin_inff();
}

// This lane's row of 8 operand registers.
__device__ __forceinline__ void load_row(bf16x8 (&f)[8], const uint16_t* p, bool valid, int hh) {
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) {
    uint4 x = make_uint4(0, 0, 0, 0);
    if (valid) x = *reinterpret_cast<const uint4*>(p + 16 * kk + 8 * hh);
    f[kk] = __builtin_bit_cast(bf16x8, x);
  }
}

__device__ __forceinline__ uint2 pack4(const f32x16& s, int x) {
  return make_uint2(pack_bf16x2(s[4 * x], s[4 * x + 1]), pack_bf16x2(s[4 * x + 2], s[4 * x + 3]));
}

// A wave's 32 rows to memory as bf16: words(d, q) are this lane's row's dims
// 32 d + 8 q + 4 (lane / 32) on.  They go through LDS of the wave's own (`mine`,
// kOutBytes), so that 16 lanes write the 256 bytes of a row (lane by lane a store
// would touch 32 rows, 8 bytes at a time: 512 pieces for 64 cache lines; the
// forward call of 512 rows x 16 heads for training took 28 us, 25 now).
// Rows [from, rows) of the 32 are written.
constexpr int kOutStride = 2 * D + 16, kOutBytes = 32 * kOutStride;
template <class Words>
__device__ __forceinline__ void store_rows(uint8_t* mine, int lane, uint16_t* to, int64_t sn, int from, int rows,
                                           Words&& words) {
  uint8_t* row = mine + (lane & 31) * kOutStride + (lane >> 5) * 8;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int q = 0; q < 4; ++q) *reinterpret_cast<uint2*>(row + 64 * d + 16 * q) = words(d, q);
  asm volatile("" ::: "memory");  // the wave's LDS operations stay in order
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const int r = 4 * u + (lane >> 4), cc = lane & 15;
    const uint4 x = *reinterpret_cast<const uint4*>(mine + r * kOutStride + 16 * cc);
    if (r >= from && r < rows) *reinterpret_cast<uint4*>(to + (int64_t)r * sn + 8 * cc) = x;
  }
  asm volatile("" ::: "memory");
}

// What rounding to bf16 left of values: kept beside outputs for
// training, so that the gradients' sums dout . o start from 16 bits of o (in a
// row that one key has most of they cancel against that key's dout . v).
__device__ __forceinline__ uint32_t left2(float a, float b, uint32_t packed) {
  return pack_bf16x2(a - __uint_as_float(packed << 16), b - __uint_as_float(packed & 0xffff0000u));
}
__device__ __forceinline__ uint2 left4(const f32x16& s, int x, uint2 packed) {
  return make_uint2(left2(s[4 * x], s[4 * x + 1], packed.x), left2(s[4 * x + 2], s[4 * x + 3], packed.y));
}

// log2 of a row's sum of exponentials; -inf for a row without keys.
__device__ __forceinline__ float log2_sum(float m, float l, float c) {
  return l > 0.0f ? m * c + log2f(l) : -__builtin_inff();
}

// A value that all lanes hold, read to the end here: left in flight into a
// loop, a load would have the loop wait for all its copies.
__device__ __forceinline__ float uniform(float x) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}
// Keeps a value where it is computed: the compiler moves what is used once to
// where it is used.
__device__ __forceinline__ void pin(float& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void pin(uint32_t& x) { asm volatile("" : "+v"(x)); }

}  // namespace
}  // namespace sol
