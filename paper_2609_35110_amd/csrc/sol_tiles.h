// Tiles of bf16 rows staged in LDS and the MFMA fragments read from them:
// shared by the linear (sol_lin_attn.hip), differential (sol_diff_attn.hip) and
// cross (sol_cross_attn.hip) attention.
#pragma once

#include <type_traits>
#include <utility>

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

// A tile of rows in LDS as the copies below leave it: blocks of 8 rows by 128
// bytes, 1 KB each, two to 8 rows, row after row, the 16-byte chunk c of row r
// at place c ^ swizzle(r) of the row's eight.  So a copy's destination is linear
// over the lanes and its source 128 consecutive bytes a row; the eight rows'
// chunks of a fragment read, and the four rows' pairs of chunks of a transpose
// read, touch no bank twice; and every fragment of a tile is one address of the
// lane's (two for the row fragments) and a constant.
constexpr int kRowBlock = 2048;         // bytes of 8 rows
constexpr int kTile32 = 4 * kRowBlock;  // bytes of 32 rows
__device__ __forceinline__ int swizzle(int r) { return (r & 2) | ((r >> 2) & 1); }
// Row fragments kk (places 16 kk + 8 (lane / 32) on of row lane % 32): even kk
// from .even, odd from .odd.
struct RowPlace {
  int even, odd;
};
__device__ __forceinline__ RowPlace row_place(int lane) {
  const int r = lane & 31, at = (r >> 3) * kRowBlock + (r & 7) * 128, f = swizzle(r) ^ (lane >> 5);
  return {at + f * 16, at + (f ^ 2) * 16};
}
__device__ __forceinline__ bf16x8 row_frag(const uint8_t* tile, const RowPlace& p, int kk) {
  return *reinterpret_cast<const bf16x8*>(tile + (kk & 1 ? p.odd : p.even) + ((kk >> 1) & 1) * 64 + (kk >> 2) * 1024);
}
__device__ __forceinline__ int col_place(int lane) {
  const int g16 = lane >> 4, i16 = lane & 15, r = 4 * (g16 >> 1) + (i16 >> 2);
  return r * 128 + ((2 * (g16 & 1) + ((i16 & 3) >> 1)) ^ swizzle(r)) * 16 + (i16 & 1) * 8;
}
// Column lane % 32 of dims 32 d on, 16 rows from 16 y on (p: tile + col_place).
__device__ __forceinline__ bf16x8 col_frag(const uint8_t* p, int y, int d) {
  const uint8_t* at = p + 2 * y * kRowBlock + (d >> 1) * 1024 + (d & 1) * 64;
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)at);
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at + kRowBlock));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Copies of 8 rows' first or last 64 elements (a block, 1 KB) by a wave straight
// into LDS: nothing passes through registers, and the wave waits for them with
// copies_landed.  base: the tile's first row; off: copy_offset, this lane's byte
// offset from there, 128 more for the second block.
__device__ __forceinline__ uint32_t copy_offset(int row, int64_t sn, int lane) {
  return (uint32_t)(row * sn * 2) + ((lane & 7) ^ swizzle(lane >> 3)) * 16;
}
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // M0 is a reserved register
__device__ __forceinline__ void copy_1k(uint32_t lds, const void* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}
// The same from an address of the lane's own.
__device__ __forceinline__ void copy_1k_from(uint32_t lds, const void* p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds), "v"(p) : "memory", "m0");
}
// 64 floats, one a lane.
__device__ __forceinline__ void copy_256(uint32_t lds, const void* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}
#pragma clang diagnostic pop
// This wave's copies but the last kLeft are in LDS, and every wave's once all
// have passed.
template <int kLeft>
__device__ __forceinline__ void copies_landed() {
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kLeft) : "memory");
}
// Every load of the wave's own is back, and the compiler knows it: one that it
// took to be in flight into a loop would cost a wait there, for the copies too,
// or one for all of the LDS reads on their way.
__device__ __forceinline__ void all_landed() { __builtin_amdgcn_s_waitcnt(0); }
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
// f(integral_constant<int, kFrom>) .. f(integral_constant<int, kTo - 1>): the
// slots of a turn, each compiled for its own place.
template <int kFrom, class F, int... I>
__device__ __forceinline__ void each_of(F& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, kFrom + I>{}), ...);
}
template <int kFrom, int kTo, class F>
__device__ __forceinline__ void each(F&& f) {
  each_of<kFrom>(f, std::make_integer_sequence<int, kTo - kFrom>{});
}
// Score MFMAs as inline assembly: their results go to VGPRs, where the
// exponentials read them (the builtin, in a kernel of more than 256 registers,
// puts every result in AGPRs, and each score would cost a move).  The compiler
// does not see that these are MFMAs: what reads or overwrites a result stands
// behind settle(), or some slots with MFMAs behind (a result is there 12 wait
// states after its MFMA).  score_a takes the second operand from AGPRs.
__device__ __forceinline__ void score_first(f32x16& d, const bf16x8& a, const bf16x8& b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(d) : "v"(a), "v"(b));
}
__device__ __forceinline__ void score(f32x16& d, const bf16x8& a, const bf16x8& b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(d) : "v"(a), "v"(b));
}
__device__ __forceinline__ void score_first_a(f32x16& d, const bf16x8& a, const bf16x8& b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(d) : "v"(a), "a"(b));
}
__device__ __forceinline__ void score_a(f32x16& d, const bf16x8& a, const bf16x8& b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(d) : "v"(a), "a"(b));
}
// Operands in AGPRs (score_a) or VGPRs (score) from here on, two wait states
// before an MFMA reads them.
__device__ __forceinline__ void hold_in_vgprs(bf16x8 (&a)[8]) {
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+v"(a[kk]));
  asm volatile("s_nop 1");
}
__device__ __forceinline__ void hold_in_agprs(bf16x8 (&a)[8]) {
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+a"(a[kk]));
  asm volatile("s_nop 1");
}
__device__ __forceinline__ void settle(f32x16& a, f32x16& b) {
  asm volatile("s_nop 7\n\ts_nop 7" : "+v"(a), "+v"(b)::"memory");
}
// Keeps what is written in this order from being moved across.
__device__ __forceinline__ void slot_end() { __builtin_amdgcn_sched_barrier(0); }

// The larger (sum) of the two lanes l and l ^ 32, in both.
__device__ __forceinline__ float both_max(float x) { return fmaxf(x, __shfl_xor(x, 32)); }
__device__ __forceinline__ float both_sum(float x) { return x + __shfl_xor(x, 32); }

}  // namespace
}  // namespace sol
