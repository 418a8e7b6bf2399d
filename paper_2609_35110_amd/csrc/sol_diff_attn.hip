// Differential attention (sol_diff_attn_fwd, _bwd): for every output head the
// difference of two softmax maps over the same values,
//   out = softmax(scale q_0 k_0^T) v - lambda softmax(scale q_1 k_1^T) v,
// query heads 2h and 2h + 1 of q being the maps of output head h.
//
// One pass over the keys with the running maximum and sum of each row and map;
// scores S^T = K Q^T and outputs O^T = V^T P^T, so that a lane owns a row: its
// maximum, sum and rescaling are the lane's own, and P as the score MFMA
// leaves it is the operand of the next.  fp32 throughout but for the operands:
// P is rounded to bf16, as the values are bf16, and its product divided by the
// sum of the rounded ones.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "sol_ops.h"
#include "sol_softmax.h"

namespace sol {
namespace {

struct Seq {
  int qlen, klen, shift;  // row i sees keys up to i + shift
};
__device__ __forceinline__ Seq sequence(const DiffShape& s, int b) {
  Seq q;
  q.qlen = s.q_lens ? min(max(s.q_lens[b], 0), s.N) : s.N;
  q.klen = s.kv_lens ? min(max(s.kv_lens[b], 0), s.M) : s.M;
  q.shift = s.causal ? q.klen - q.qlen : s.M;
  return q;
}

// out and out2 of two dims from `d` of row (b, h, n).
__device__ __forceinline__ void store_row2(const DiffFwd& A, int b, int h, int n, int d, float lam, const float2 (&o)[2]) {
  const float2 y = make_float2(__builtin_fmaf(-lam, o[1].x, o[0].x), __builtin_fmaf(-lam, o[1].y, o[0].y));
  const uint32_t w = pack_bf16x2(y.x, y.y);
  *reinterpret_cast<uint32_t*>(A.out.p + b * A.out.sb + h * A.out.sh + (int64_t)n * A.out.sn + d) = w;
  if (A.out2) {
    uint16_t* p = A.out2 + (((int64_t)b * A.s.H + h) * A.s.N + n) * (3 * D) + d;
    const uint32_t w1 = pack_bf16x2(o[1].x, o[1].y);
    *reinterpret_cast<uint32_t*>(p) = w1;
    *reinterpret_cast<uint32_t*>(p + D) = left2(o[1].x, o[1].y, w1);
    *reinterpret_cast<uint32_t*>(p + 2 * D) = left2(y.x, y.y, w);
  }
}

// Results of pieces of the keys, to be joined: o fp32 [piece][map][row][128],
// then the log2 of the sums that o was divided by, [piece][map][row], and of the
// exact ones (for training), for `rows` rows: those of the tiles that
// are split (tile after tile), or, where the few-row kernel splits, all
// [B][H][N].
struct Parts {
  float *o, *l, *exact;
  int64_t rows;
};
__device__ __forceinline__ Parts parts_of(float* ws, int64_t rows, int pieces) {
  return {ws, ws + rows * 2 * pieces * D, ws + rows * 2 * pieces * (D + 1), rows};
}

// Tiles of 128 rows (keys) of the batch's slabs, `heads` per sequence, in the
// order that workgroups take them, a run of consecutive ones to an XCD:
//  - slab after slab, sequence after sequence;
//  - where lengths differ, head after head, so that every XCD has some of each
//    sequence (4 sequences of 2,047 to 511 rows, 16 heads: forward 227 -> 142 us,
//    gradients 729 -> 421);
//  - by rank under a causal mask, the longest tiles of all slabs first, every
//    eighth to an XCD, so that the short ones fill what the long ones leave
//    (12,480 rows x 3 heads: forward 413 -> 298 us, gradients 890 -> 667; 4,096 x
//    24: 241 -> 220, 628 -> 612).  Not where lengths differ and an XCD has two
//    slabs or more: there one head at a time in its L2 is worth more (4,097 and
//    2,048 rows x 8 heads: 113 us head after head, 136 by rank).
__host__ __device__ inline bool by_rank(const DiffShape& s, int heads) {
  return s.causal && (!(s.q_lens || s.kv_lens) || s.B * heads < 16);
}
struct SlabTile {
  int b, h, rank;
};
__device__ __forceinline__ SlabTile slab_tile(int i, int per_slab, int heads, const DiffShape& s) {
  if (by_rank(s, heads)) {
    const int slabs = s.B * heads, rank = i / slabs, slab = i - rank * slabs;
    return {slab / heads, slab % heads, rank};
  }
  const int slab = i / per_slab, rank = i - slab * per_slab;
  if (s.q_lens || s.kv_lens) return {slab % s.B, slab / s.B, rank};
  return {slab / heads, slab % heads, rank};
}
// The tile and piece of a workgroup: tiles [0, full) whole, the rest in pieces.
struct Piece {
  int tile, piece, pieces;
};
__device__ __forceinline__ Piece piece_of(int wg, int tiles, const DiffTiles& p, bool by_rank) {
  if (wg < p.full) return {by_rank ? wg : xcd_local_id(wg, p.full), 0, 1};
  const int id = by_rank ? wg - p.full : xcd_local_id(wg - p.full, (tiles - p.full) * p.pieces);
  return {p.full + id / p.pieces, id % p.pieces, p.pieces};
}
// The row tiles: a head's last rows first (under a causal mask the longest), whole
// ones from its end, so that the odd rows are the first ones, which see the fewest
// keys (2 x 4,097 rows, 8 heads, causal, for training: forward 154 us instead of 161
// with all the keys for a tile of one row).  The last tile's first rows may be below 0.
struct RowTile {
  int b, h, row0;
};
__device__ __forceinline__ RowTile row_tile(int tile, const DiffShape& s) {
  const int per_head = (s.N + kDiffRows - 1) / kDiffRows;
  const SlabTile at = slab_tile(tile, per_head, s.H, s);
  return {at.b, at.h, s.N - (at.rank + 1) * kDiffRows};
}
__host__ __device__ inline int row_tiles_of(const DiffShape& s) {
  return s.B * s.H * ((s.N + kDiffRows - 1) / kDiffRows);
}

// ------------------------------------------------------------------- forward

// These kernels are one wave a SIMD, whose MFMAs, exponentials and LDS reads
// have to overlap inside the wave: a turn of the loop is a list of slots, each
// an MFMA, the LDS read of a fragment some slots on and a share of the
// arithmetic on scores that are done, and nothing moves between slots.  Tiles
// come through LDS in a ring of four, copied two turns ahead.

constexpr int kRing = 4;

// 128 rows of one head, 32 a wave, both maps in the wave (a fragment of V, and
// of a shared K, is read once for two MFMAs).  Turn t: the products P V of tile
// t - 1, under them map 0's exponentials of tile t; then the scores of tile
// t + 1, under them map 1's.
//
// A row is held to the maximum of its first tile: P and the sums have 8 exponent
// bits, so scores far above it cost no precision, and most rows' stay within a
// few binades.  A row whose P add up to more than 2^80 (55 above it in the
// exponent), or whose products with the values leave fp32, has its workgroup walk the
// keys again, held to the rows' own maxima, found by a walk for scores alone.
//
// 12,480 rows x 24 heads: 3.25 to 3.5 ms by box and what ran before, 1,100 to 1,180
// TFLOP/s, 84 to 90 % of a large bf16 product's rate here; the matrix cores are busy
// 60 % of the cycles at 1.7 GHz, which the chip's power sets (4.3 vector instructions
// an MFMA).  For training, with the second sum and two more outputs, 24 heads take
// 3,361 us instead of 3,250; causal 2 x 4,097 rows x 8 heads 163 instead of 147.
constexpr int kFwdKeys = 32;
constexpr float kTooMuch = 1.2089258e24f;
template <bool kShared, bool kTrain>
__global__ __launch_bounds__(256, 1) void diff_fwd_kernel(DiffFwd A, DiffTiles plan) {
  constexpr int kTiles = kShared ? 2 : 3;  // K (of each map), V
  constexpr int kV = kTiles - 1;
  constexpr int kKFrags = kShared ? 8 : 16, kFrags = 8 + kKFrags, kAhead = 6, kHold = 8;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kRing][kTiles][kTile32];
  lds_poison(lds, sizeof(lds));
  lds_poison_done();
  const DiffShape& s = A.s;
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  const Piece pc = piece_of(blockIdx.x, row_tiles_of(s), plan, by_rank(s, s.H));
  const RowTile rt = row_tile(pc.tile, s);
  const int b = rt.b, h = rt.h, row0 = rt.row0;
  const Seq sq = sequence(s, b);
  if (row0 >= sq.qlen) return;
  const int per = s.H / s.Hv, hv = h / per;
  const int row = row0 + 32 * wave + l32;
  const bool valid = row >= 0 && row < sq.qlen;
  const float c = s.scale * kLog2e;

  const uint16_t* k0 = A.k.p + b * A.k.sb + (kShared ? hv : 2 * hv) * A.k.sh;
  const uint16_t* v0 = A.v.p + b * A.v.sb + hv * A.v.sh;
  bf16x8 qf[2][8];
  load_row(qf[0], A.q.p + b * A.q.sb + 2 * h * A.q.sh + (int64_t)row * A.q.sn, valid, hh);
  load_row(qf[1], A.q.p + b * A.q.sb + (2 * h + 1) * A.q.sh + (int64_t)row * A.q.sn, valid, hh);

  const int last = min(row + sq.shift, sq.klen - 1);  // of this lane's row
  const int last_row = min(row0 + kDiffRows, sq.qlen) - 1;
  const int2 range = split_keys(max(min(last_row + sq.shift, sq.klen - 1) + 1, 0), pc.piece, pc.pieces, kFwdKeys);
  const int turns = (range.y - range.x + kFwdKeys - 1) / kFwdKeys;
  const int all_to = min(row0 + 32 * wave + sq.shift, sq.klen - 1);  // every row of the wave sees these

  const uint32_t at0 = lds_address(&lds[0][0][0]) + wave * kRowBlock;
  const int copy_row = 8 * wave + (lane >> 3);
  // Tile after tile into place `place` of the ring, one kilobyte at a time; past
  // the last tile it comes again, and is not used.
  constexpr int kCopies = 2 * kTiles;
  struct Copy {
    const uint16_t *k, *v;
    int key;
    uint32_t to, ok, ov;
  } cp_ = {};
  auto copy_start = [&](int i, int place) __attribute__((always_inline)) {
    if (i == 0) {
      cp_.key = range.x;
      cp_.k = k0 + (int64_t)range.x * A.k.sn;
      cp_.v = v0 + (int64_t)range.x * A.v.sn;
      cp_.ok = copy_offset(copy_row, A.k.sn, lane);
      cp_.ov = copy_offset(copy_row, A.v.sn, lane);
    }
    const bool on = i > 0 && i < turns;
    cp_.k += on ? kFwdKeys * A.k.sn : 0;
    cp_.v += on ? kFwdKeys * A.v.sn : 0;
    cp_.key += on ? kFwdKeys : 0;
    cp_.to = __builtin_amdgcn_readfirstlane(at0 + (place % kRing) * (kTiles * kTile32));
    if (cp_.key + kFwdKeys > sq.klen) {  // keys past the sequence: its last key again (their scores are masked)
      const int r = min(copy_row, sq.klen - 1 - cp_.key);
      cp_.ok = copy_offset(r, A.k.sn, lane);
      cp_.ov = copy_offset(r, A.v.sn, lane);
    }
  };
  auto copy_part = [&](int n) __attribute__((always_inline)) {
    const uint16_t* p = n / 2 == kV ? cp_.v : n / 2 == 0 ? cp_.k : cp_.k + A.k.sh;
    copy_1k(cp_.to + n / 2 * kTile32 + n % 2 * 1024, p, (n / 2 == kV ? cp_.ov : cp_.ok) + n % 2 * 128);
  };
  auto copy = [&](int i, int place) __attribute__((always_inline)) {
    copy_start(i, place);
#pragma unroll
    for (int n = 0; n < kCopies; ++n) copy_part(n);
  };

  struct Tile {
    f32x16 s[2];         // scores
    uint32_t pw[2][8];   // P, packed
  } ta, tb;
  MapRows x[2];
  clear(x[0]);
  clear(x[1]);
  float mc[2];
  bf16x8 ring[kHold];
  const RowPlace rp = row_place(lane);
  const int cp = col_place(lane);
  // the fragments of a turn in order: V of tile t - 1, then K of tile t + 1
  auto fragment = [&](int f, const uint8_t* then, const uint8_t* next) __attribute__((always_inline)) {
    if (f < 8) return col_frag(then + kV * kTile32 + cp, f >> 2, f & 3);
    const int j = f - 8;
    return row_frag(next + (kShared ? 0 : (j & 1) * kTile32), rp, kShared ? j : j >> 1);
  };
  auto mask_tile = [&](Tile& now, int i) __attribute__((always_inline)) {
    const int key = range.x + i * kFwdKeys;
    if (key + kFwdKeys - 1 > all_to || i >= turns) {
      const int to = i < turns ? last : -1;  // (past the last tile: none)
      settle(now.s[0], now.s[1]);
      mask(now.s[0], key + 4 * hh, to);
      mask(now.s[1], key + 4 * hh, to);
    }
  };
  // one exponential; its pair is summed and packed with the next one's (an
  // exponential's result is not there at once)
  float e[2];
  auto take = [&](Tile& now, int m, int r) __attribute__((always_inline)) {  // rows r, r + 1
    if (kTrain) x[m].exact += e[0];
    now.pw[m][r >> 1] = pack_bf16x2(e[0], e[1]);
    if (kTrain) x[m].exact += e[1];
    pin(now.pw[m][r >> 1]);
    x[m].l = add_bf16x2(now.pw[m][r >> 1], x[m].l);
    pin(x[m].l);
    if (kTrain) pin(x[m].exact);
  };
  auto exponential = [&](Tile& now, int m, int r) __attribute__((always_inline)) {
    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(now.s[m][r], c, -mc[m]));
    if (r % 2 == 0 && r > 0) take(now, m, r - 2);
    if (r == 0 && m == 1) take(now, 0, 14);
    e[r & 1] = p;
    pin(e[r & 1]);
  };
  auto operand = [&](const Tile& z, int m, int y) __attribute__((always_inline)) {
    return __builtin_bit_cast(bf16x8, make_uint4(z.pw[m][4 * y], z.pw[m][4 * y + 1], z.pw[m][4 * y + 2], z.pw[m][4 * y + 3]));
  };
  // old: tile i - 1's P, and room for tile i + 1's scores
  auto turn = [&](int i, Tile& now, Tile& old) __attribute__((always_inline)) {
    const uint8_t* to = &lds[(i + kRing - 1) % kRing][0][0];
    const uint8_t* tn = &lds[i % kRing][0][0];
    const uint8_t* next = &lds[(i + 1) % kRing][0][0];
    mask_tile(now, i);
#pragma unroll
    for (int d = 0; d < 4; ++d) asm volatile("" : "+a"(x[0].o[d]), "+a"(x[1].o[d]));
    hold_in_agprs(qf[0]);
    hold_in_agprs(qf[1]);
    each<0, 32>([&](auto slot) __attribute__((always_inline)) {
      constexpr int j = slot.value;
      if constexpr (j == 2) {
        copies_landed<0>();
        copy_start(i + 2, i + 2);
        slot_end();
      }
      if constexpr (j >= 3 && j < 3 + kCopies) copy_part(j - 3);
      constexpr bool kFirstUse = j < 16 ? j % 2 == 0 : !kShared || j % 2 == 0;
      constexpr int f = j < 16 ? j / 2 : 8 + (kShared ? (j - 16) / 2 : j - 16);
      if constexpr (j < 16) {
        constexpr int m = j & 1, d = (j >> 1) & 3, y = j >> 3;
        x[m].o[d] = mfma(ring[f % kHold], operand(old, m, y), x[m].o[d]);
      } else {
        constexpr int m = j & 1, kk = (j - 16) >> 1;
        if constexpr (kk == 0) score_first_a(old.s[m], ring[f % kHold], qf[m][kk]);
        else score_a(old.s[m], ring[f % kHold], qf[m][kk]);
      }
      if constexpr (kFirstUse) {
        constexpr int g = f + kAhead;
        ring[g % kHold] = g < kFrags ? fragment(g, to, next) : fragment(g - kFrags, tn, nullptr);
      }
      if constexpr (j >= 2 && j < 16) {
#pragma unroll
        for (int e = (j - 2) * 8 / 7; e < (j - 1) * 8 / 7; ++e) exponential(now, 0, e);
      }
      if constexpr (j >= 16) exponential(now, 1, j - 16);
      slot_end();
    });
    take(now, 1, 14);
  };
  // scores of tile i, which is in the ring's place 0, all at once
  auto scores_of = [&](Tile& z, int i) __attribute__((always_inline)) {
    const uint8_t* tk = &lds[0][0][0];
    hold_in_agprs(qf[0]);
    hold_in_agprs(qf[1]);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const bf16x8 f0 = row_frag(tk, rp, kk), f1 = kShared ? f0 : row_frag(tk + kTile32, rp, kk);
      if (kk == 0) {
        score_first_a(z.s[0], f0, qf[0][kk]);
        score_first_a(z.s[1], f1, qf[1][kk]);
      } else {
        score_a(z.s[0], f0, qf[0][kk]);
        score_a(z.s[1], f1, qf[1][kk]);
      }
    }
    settle(z.s[0], z.s[1]);
    mask_tile(z, i);
  };
  auto raise = [&](const Tile& z) __attribute__((always_inline)) {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float top = z.s[m][0];
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(top, z.s[m][r]);
      x[m].m = fmaxf(x[m].m, both_max(top));
    }
  };
  // Large values under P that pass 1 may leave fp32 with sums that stay below 2^80:
  // looked for in waves where a row's P add up to more than its keys could at 1.
  auto not_finite = [&]() __attribute__((always_inline)) {
    if (!__any(x[0].l > (float)SOL_MAX_TOKENS || x[1].l > (float)SOL_MAX_TOKENS)) return false;
    uint32_t top = 0;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        top = max(top, max(__float_as_uint(x[0].o[d][r]) & 0x7fffffffu, __float_as_uint(x[1].o[d][r]) & 0x7fffffffu));
    return top >= 0x7f800000u;
  };
  for (int attempt = 0; turns > 0; ++attempt) {
    copy(0, 0);
    copy(0, kRing - 1);  // turn 0's products, of P = 0
    copies_landed<0>();
    all_landed();
    copy(1, 1);
    scores_of(ta, 0);
    raise(ta);
    mc[0] = x[0].m * c;
    mc[1] = x[1].m * c;
#pragma unroll
    for (int w = 0; w < 8; ++w) tb.pw[0][w] = tb.pw[1][w] = 0;
#pragma unroll
    for (int f = 0; f < kAhead; ++f) ring[f] = fragment(f, &lds[kRing - 1][0][0], nullptr);
    for (int i = 0; i <= turns; i += 2) {
      turn(i, ta, tb);
      turn(i + 1, tb, ta);
    }
    copies_landed<0>();  // none is under way when the wave ends
    if (attempt || !__syncthreads_or(!(x[0].l < kTooMuch && x[1].l < kTooMuch) || not_finite())) break;
    clear(x[0]);
    clear(x[1]);
    for (int i = 0; i < turns; ++i) {
      __syncthreads();
      copy(i, 0);
      copies_landed<0>();
      scores_of(ta, i);
      raise(ta);
    }
    __syncthreads();
  }

  float l2[2], exact2[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const float l = both_sum(x[m].l);
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    l2[m] = log2_sum(x[m].m, l, c);
    if (kTrain) exact2[m] = log2_sum(x[m].m, both_sum(x[m].exact), c);
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[m].o[d][r] *= inv;
  }
  if (pc.pieces > 1) {
    if (!valid) return;
    const Parts p = parts_of(A.ws, (int64_t)(row_tiles_of(s) - plan.full) * kDiffRows, pc.pieces);
    const int64_t pr = (int64_t)(pc.tile - plan.full) * kDiffRows + row - row0;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int64_t am = (2 * pc.piece + m) * p.rows + pr;
      float* o = p.o + am * D + 4 * hh;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(o + 32 * d + 8 * q) = make_float4(
              x[m].o[d][4 * q], x[m].o[d][4 * q + 1], x[m].o[d][4 * q + 2], x[m].o[d][4 * q + 3]);
      if (hh == 0) p.l[am] = l2[m];
      if (kTrain && hh == 0) p.exact[am] = exact2[m];
    }
    return;
  }
  if (kTrain && valid && hh == 0) {
    const int64_t at = ((int64_t)(b * 2 * s.H + 2 * h)) * s.N + row;
    A.lse[at] = exact2[0] * kLn2;
    A.lse[at + s.N] = exact2[1] * kLn2;
  }
  const float lam = s.lambda[h];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) x[0].o[d][r] = __builtin_fmaf(-lam, x[1].o[d][r], x[0].o[d][r]);
  uint8_t* mine = &lds[0][0][0] + wave * kOutBytes;
  const int first = row0 + 32 * wave, rows = sq.qlen - first;
  store_rows(mine, lane, A.out.p + b * A.out.sb + h * A.out.sh + (int64_t)first * A.out.sn, A.out.sn, -first, rows,
             [&](int d, int q) { return pack4(x[0].o[d], q); });
  if (kTrain) {
    uint16_t* o2 = A.out2 + (((int64_t)b * s.H + h) * s.N + first) * (3 * D);
    store_rows(mine, lane, o2, 3 * D, -first, rows, [&](int d, int q) { return pack4(x[1].o[d], q); });
    store_rows(mine, lane, o2 + D, 3 * D, -first, rows,
               [&](int d, int q) { return left4(x[1].o[d], q, pack4(x[1].o[d], q)); });
    store_rows(mine, lane, o2 + 2 * D, 3 * D, -first, rows,
               [&](int d, int q) { return left4(x[0].o[d], q, pack4(x[0].o[d], q)); });
  }
}

// Groups of rows of one value head's heads in the few-row kernel.
__host__ __device__ inline int few_groups(const DiffShape& s) {
  return (int)(((int64_t)(s.H / s.Hv) * s.N + kFewRows - 1) / kFewRows);
}
// Few rows over many keys (a token or some drafted ones over a cache): the rows
// of all heads that share a value head -- row r is token r % N of head
// hv per + r / N -- in groups of one wave's 32, a workgroup each (the tile kernel
// would give every head a tile of 128).  The keys' bytes bound it, so each wave
// of the workgroup walks every fourth block of 32 keys with both maps on its
// own, through LDS of its own (no barriers), the next block's bytes in flight
// in its registers; the four waves' rows are joined at the end.  5.7 to 5.9 TB/s over
// 111,600 keys of 40 heads (580 to 600 us), 5.3 over 32 caches of 256 to 8,192 (104 us);
// P in two bf16 parts, as exact as the outputs' own rounding, costs 2 to 12 % there.
template <bool kShared>
__global__ __launch_bounds__(256, 1) void diff_few_kernel(DiffFwd A, int nsplit) {
  constexpr int kBlock = 32, kWaves = 4;
  constexpr int kTileElems = kBlock * kStride;
  constexpr int kKTiles = kShared ? 1 : 2;
  constexpr int kRow = D + 4;
  struct Joined {
    float o[kWaves][2][kFewRows][kRow];
    float m[kWaves][2][kFewRows], l[kWaves][2][kFewRows], exact[kWaves][2][kFewRows];
  };
  union Lds {
    uint16_t tiles[kWaves][(kKTiles + 1) * kTileElems];
    Joined j;
  };
  __shared__ __attribute__((aligned(16))) Lds lds;
  lds_poison(&lds, sizeof(lds));
  lds_poison_done();
  const DiffShape& s = A.s;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  // (sequence, value head, piece of the keys) after another over the XCDs, but the
  // groups of rows that read the same keys on one, side by side
  const int per = s.H / s.Hv, groups = few_groups(s);
  int id = blockIdx.x / (8 * groups) * 8 + blockIdx.x % 8;
  const int row_base = blockIdx.x / 8 % groups * kFewRows, n_rows = min(per * s.N - row_base, kFewRows);
  if (id >= s.B * s.Hv * nsplit) return;
  const int split = id % nsplit;
  id /= nsplit;
  const int hv = id % s.Hv, b = id / s.Hv;
  const Seq sq = sequence(s, b);
  const float c = s.scale * kLog2e;
  const int my = row_base + min(l32, n_rows - 1);
  const int h = hv * per + my / s.N, row = my % s.N;
  const bool valid = l32 < n_rows && row < sq.qlen;
  const int last = min(row + sq.shift, sq.klen - 1);
  const int all_to = min(sq.shift, sq.klen - 1);  // the last key that every row sees

  const uint16_t* k0 = A.k.p + b * A.k.sb + (kShared ? hv : 2 * hv) * A.k.sh;
  const uint16_t* k1 = k0 + (kShared ? 0 : A.k.sh);
  const uint16_t* v = A.v.p + b * A.v.sb + hv * A.v.sh;
  bf16x8 qf[2][8];
#pragma unroll
  for (int m = 0; m < 2; ++m)
    load_row(qf[m], A.q.p + b * A.q.sb + (2 * h + m) * A.q.sh + (int64_t)row * A.q.sn, valid, hh);

  const int2 range = split_keys(sq.klen, split, nsplit, kBlock * kWaves);
  MapRows x[2];
  clear(x[0]);
  clear(x[1]);
  uint16_t* tk = lds.tiles[wave];
  uint16_t* tv = tk + kKTiles * kTileElems;
  const int tr = column_offset(lane);
  Stage<kBlock, 64> sk0, sk1, sv;
  auto load = [&](int key) __attribute__((always_inline)) {
    sk0.load(k0, A.k.sn, key, range.y, lane);
    if (!kShared) sk1.load(k1, A.k.sn, key, range.y, lane);
    sv.load(v, A.v.sn, key, range.y, lane);
  };
  int key = range.x + wave * kBlock;
  load(key);
  for (; key < range.y; key += kBlock * kWaves) {
    sk0.store(tk, lane);
    if (!kShared) sk1.store(tk + kTileElems, lane);
    sv.store(tv, lane);
    // the wave's own LDS: its reads below follow its writes above, and those
    // the reads of the turn before (a wave's LDS operations stay in order; this
    // keeps the compiler from moving them past each other)
    asm volatile("" ::: "memory");
    load(key + kBlock * kWaves);
    f32x16 sc[2][1] = {{scores(tk, qf[0], lane)}, {scores(kShared ? tk : tk + kTileElems, qf[1], lane)}};
    if (key + kBlock - 1 > all_to) {
      mask(sc[0][0], key + 4 * hh, last);
      mask(sc[1][0], key + 4 * hh, last);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      raise_max(x[m], sc[m], c);
      exponentials(x[m], sc[m][0], c);
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const bf16x8 p0 = operand8(sc[0][0], y), p1 = operand8(sc[1][0], y);
      x[0].l = add_bf16x8(p0, x[0].l);
      x[1].l = add_bf16x8(p1, x[1].l);
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const bf16x8 vf = column8(tv + 16 * y * kStride + 32 * d + tr);
        x[0].o[d] = mfma(vf, p0, x[0].o[d]);
        x[1].o[d] = mfma(vf, p1, x[1].o[d]);
      }
    }
    asm volatile("" ::: "memory");
  }

  // join the waves' rows
  __syncthreads();
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const float l = both_sum(x[m].l), exact = both_sum(x[m].exact);
    if (l32 < n_rows) {
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(&lds.j.o[wave][m][l32][32 * d + 8 * q + 4 * hh]) =
              make_float4(x[m].o[d][4 * q], x[m].o[d][4 * q + 1], x[m].o[d][4 * q + 2], x[m].o[d][4 * q + 3]);
      if (hh == 0) {
        lds.j.m[wave][m][l32] = x[m].m;
        lds.j.l[wave][m][l32] = l;
        lds.j.exact[wave][m][l32] = exact;
      }
    }
  }
  __syncthreads();
  const Parts p = parts_of(A.ws, (int64_t)s.B * s.H * s.N, nsplit);
  // one pair of dims of one row a thread and turn
  for (int i = t; i < n_rows * (D / 2); i += 256) {
    const int r = i / (D / 2), d = 2 * (i % (D / 2));
    const int hr = hv * per + (row_base + r) / s.N, n = (row_base + r) % s.N;
    if (n >= sq.qlen) continue;
    float2 o[2];
    float l2[2], exact2[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float top = kNoMax, sum = 0.0f, exact = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds.j.m[w][m][r]);
      o[m] = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f((lds.j.m[w][m][r] - top) * c);
        sum = __builtin_fmaf(f, lds.j.l[w][m][r], sum);
        exact = __builtin_fmaf(f, lds.j.exact[w][m][r], exact);
        o[m].x = __builtin_fmaf(f, lds.j.o[w][m][r][d], o[m].x);
        o[m].y = __builtin_fmaf(f, lds.j.o[w][m][r][d + 1], o[m].y);
      }
      const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
      o[m].x *= inv;
      o[m].y *= inv;
      l2[m] = log2_sum(top, sum, c);
      exact2[m] = log2_sum(top, exact, c);
    }
    const int64_t at = ((int64_t)(b * 2 * s.H + 2 * hr)) * s.N + n;
    if (nsplit > 1) {
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const int64_t am = (2 * split + m) * p.rows + ((int64_t)b * s.H + hr) * s.N + n;
        *reinterpret_cast<float2*>(p.o + am * D + d) = o[m];
        if (d == 0) p.l[am] = l2[m];
        if (d == 0 && A.lse) p.exact[am] = exact2[m];
      }
    } else {
      store_row2(A, b, hr, n, d, s.lambda[hr], o);
      if (A.lse && d == 0) {
        A.lse[at] = exact2[0] * kLn2;
        A.lse[at + s.N] = exact2[1] * kLn2;
      }
    }
  }
}

// The pieces' results joined: a wave takes a row of an output head, two dims a
// lane, both maps; of few rows, which have many pieces, four waves do.  Bound by its
// bytes and, of few rows, by latency: 5 to 13 us in the calls above.
template <bool kFew>
__global__ __launch_bounds__(256) void diff_join_kernel(DiffFwd A, DiffTiles plan) {
  __shared__ float2 of[kFew ? 8 : 1][64];
  __shared__ float sums[kFew ? 8 : 1][3];
  lds_poison(of, sizeof(of));
  lds_poison(sums, sizeof(sums));
  lds_poison_done();
  const DiffShape& s = A.s;
  const int64_t rows = kFew ? (int64_t)s.B * s.H * s.N : (int64_t)(row_tiles_of(s) - plan.full) * kDiffRows;
  constexpr int kStep = kFew ? 4 : 1;  // pieces: every fourth a wave, or all
  const int wave = threadIdx.x >> 6;
  const int64_t i = kFew ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
  if (i >= rows) return;
  const int lane = threadIdx.x & 63;
  int b, h, n;
  if (kFew) {
    n = (int)(i % s.N);
    const int bh = (int)(i / s.N);
    h = bh % s.H;
    b = bh / s.H;
  } else {
    const RowTile rt = row_tile(plan.full + (int)(i / kDiffRows), s);
    b = rt.b;
    h = rt.h;
    n = rt.row0 + (int)(i % kDiffRows);
  }
  if (n < 0 || n >= sequence(s, b).qlen) return;
  const Parts p = parts_of(A.ws, rows, plan.pieces);
  float2 o[2];
  float exact2[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    float top = kNoMax, sum = 0.0f, exact = 0.0f;
    // (loads of eight pieces at a time)
#pragma unroll 8
    for (int u = kFew ? wave : 0; u < plan.pieces; u += kStep) top = fmaxf(top, p.l[(2 * u + m) * rows + i]);
    o[m] = make_float2(0.0f, 0.0f);
#pragma unroll 8
    for (int u = kFew ? wave : 0; u < plan.pieces; u += kStep) {
      const int64_t am = (2 * u + m) * rows + i;
      const float f = __builtin_amdgcn_exp2f(p.l[am] - top);
      const float2 x = *reinterpret_cast<const float2*>(p.o + am * D + 2 * lane);
      sum += f;
      if (A.lse) exact += __builtin_amdgcn_exp2f(p.exact[am] - top);
      o[m].x = __builtin_fmaf(f, x.x, o[m].x);
      o[m].y = __builtin_fmaf(f, x.y, o[m].y);
    }
    if (kFew) {  // the four waves' parts
      const int at = wave * 2 + m;
      of[at][lane] = o[m];
      if (lane == 0) sums[at][0] = top, sums[at][1] = sum, sums[at][2] = exact;
      __syncthreads();
      top = fmaxf(fmaxf(sums[m][0], sums[2 + m][0]), fmaxf(sums[4 + m][0], sums[6 + m][0]));
      sum = exact = 0.0f;
      o[m] = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(sums[2 * w + m][0] - top);
        sum = __builtin_fmaf(f, sums[2 * w + m][1], sum);
        exact = __builtin_fmaf(f, sums[2 * w + m][2], exact);
        o[m].x = __builtin_fmaf(f, of[2 * w + m][lane].x, o[m].x);
        o[m].y = __builtin_fmaf(f, of[2 * w + m][lane].y, o[m].y);
      }
    }
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    o[m].x *= inv;
    o[m].y *= inv;
    exact2[m] = sum > 0.0f ? top + log2f(exact) : -__builtin_inff();
  }
  if (kFew && wave) return;
  store_row2(A, b, h, n, 2 * lane, s.lambda[h], o);
  if (A.lse && lane < 2) A.lse[((int64_t)(b * 2 * s.H + 2 * h) + lane) * s.N + n] = (lane ? exact2[1] : exact2[0]) * kLn2;
}

// ------------------------------------------------------------------ backward
//
// With X = dout v^T, P_s the maps and delta_s = dout . o_s of a row,
//   dS_0 = P_0 (X - delta_0),  dS_1 = -lambda P_1 (X - delta_1),
//   dq_s = scale dS_s k_s,  dk_s = scale dS_s^T q_s,
//   dv = (P_0 - lambda P_1)^T dout,  dlambda = - sum P_1 X.
// P is found again from the rows' log sums.  dS and P_0 - lambda P_1 are rounded to
// bf16 for their products with k, q and dout, which are bf16: a result's error is its
// terms' roundings and its own, of one size (0.0024 of its norm together).  Two
// halves, one that owns rows (dq) and one that owns keys (dk, dv, dlambda): no
// atomics, and every sum in a fixed order.

// What the backward kernels know of a row, 32 rows together: kStatLse0, kStatLse1:
// -lse / scale of the maps, which added to raw scores and scaled gives log2 P
// (-inf, and so P = 0, where the row has no keys or is not the sequence's);
// kStatDelta0: -delta_0; kStatStep: delta_0 - delta_1; 32 floats each.  Reading
// dout, out and out2 bounds it: 12,480 rows x 3 heads 10 us, 4.8 TB/s.
constexpr int kBwdRows = 32;
constexpr int kStatFloats = 4 * kBwdRows;
enum { kStatLse0 = 0, kStatLse1 = kBwdRows, kStatDelta0 = 2 * kBwdRows, kStatStep = 3 * kBwdRows };

__global__ __launch_bounds__(16 * kBwdRows) void diff_stats_kernel(DiffBwd A) {
  __shared__ float second[kBwdRows];  // delta_1 of the rows
  lds_poison(second, sizeof(second));
  lds_poison_done();
  const DiffShape& s = A.s;
  const int row_tiles = (s.N + kBwdRows - 1) / kBwdRows;
  const int r = threadIdx.x >> 4, cc = threadIdx.x & 15;
  const int n = (int)(blockIdx.x % row_tiles) * kBwdRows + r;
  const int bh = blockIdx.x / row_tiles, h = bh % s.H, b = bh / s.H;
  const bool valid = n < sequence(s, b).qlen;
  float d0 = 0.0f, d1 = 0.0f;
  if (valid) {
    float o[8], o1[8], g[8], left[8];
    auto load = [](float (&f)[8], const uint16_t* p) { unpack_bf16x8(*reinterpret_cast<const uint4*>(p), f); };
    load(o, A.out.p + b * A.out.sb + h * A.out.sh + (int64_t)n * A.out.sn + 8 * cc);
    load(g, A.dout.p + b * A.dout.sb + h * A.dout.sh + (int64_t)n * A.dout.sn + 8 * cc);
    const uint16_t* p = A.out2 + ((int64_t)bh * s.N + n) * (3 * D) + 8 * cc;
    load(o1, p);
    load(left, p + D);
#pragma unroll
    for (int u = 0; u < 8; ++u) o1[u] += left[u];
    load(left, p + 2 * D);
#pragma unroll
    for (int u = 0; u < 8; ++u) o[u] += left[u];
    const float lam = s.lambda[h];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      d0 = __builtin_fmaf(g[u], __builtin_fmaf(lam, o1[u], o[u]), d0);
      d1 = __builtin_fmaf(g[u], o1[u], d1);
    }
  }
#pragma unroll
  for (int m = 1; m < 16; m <<= 1) {
    d0 += __shfl_xor(d0, m);
    d1 += __shfl_xor(d1, m);
  }
  if (cc < 2) {
    const float lse = valid ? A.lse[((int64_t)bh * 2 + cc) * s.N + n] : 0.0f;
    const bool some = valid && lse > -3e38f;
    float* st = A.stats + (int64_t)blockIdx.x * kStatFloats + r;
    st[cc ? kStatLse1 : kStatLse0] = some ? -lse / s.scale : -__builtin_inff();
    st[cc ? kStatStep : kStatDelta0] = !some ? 0.0f : cc ? d0 - d1 : -d0;
    if (cc) second[r] = some ? d1 : 0.0f;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    float x = 0.0f;
    for (int i = 0; i < kBwdRows; ++i) x += second[i];
    A.delta[blockIdx.x] = x;
  }
}

// A backward turn t finds the scores and X of tile t, the exponentials of tile t
// (from the slot where its scores are done), what is left of tile t - 1 to its
// operands, and the gradient products of tile t - 1.  A turn's slot j reads the
// fragment of slot j + kAhead (kAhead a divisor of the list's length: a
// fragment's register is the same in every turn); the barrier stands where the
// last eight slots begin, so that the next tile's first fragments are read
// before the turn ends.
struct Scores {
  f32x16 s[2], x;  // scores of the maps, X
  float p[2][16];  // P of the maps
};

// dq of 128 rows of one head, both maps in a wave (X is found once): 32 rows a
// wave over all the keys they see.
constexpr int kDqKeys = 32;
template <bool kShared>
__device__ __forceinline__ void dq_of(const DiffBwd& A, uint8_t (*lds)[kShared ? 2 : 3][kTile32], int wg) {
  constexpr int kTiles = kShared ? 2 : 3;  // K (of each map), V
  constexpr int kV = kTiles - 1;
  constexpr int kAhead = 8;
  const DiffShape& s = A.s;
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  const Piece pc = piece_of(wg, row_tiles_of(s), A.plan, by_rank(s, s.H));
  const RowTile rt = row_tile(pc.tile, s);
  const int b = rt.b, h = rt.h, row0 = rt.row0;
  const Seq sq = sequence(s, b);
  const int per = s.H / s.Hv, hv = h / per;
  const int row = row0 + 32 * wave + l32;
  const bool valid = row >= 0 && row < sq.qlen;
  const float c = s.scale * kLog2e, lam = s.lambda[h];

  const uint16_t* k0 = A.k.p + b * A.k.sb + (kShared ? hv : 2 * hv) * A.k.sh;
  const uint16_t* v0 = A.v.p + b * A.v.sb + hv * A.v.sh;
  bf16x8 qf[2][8], gf[8];
  load_row(qf[0], A.q.p + b * A.q.sb + 2 * h * A.q.sh + (int64_t)row * A.q.sn, valid, hh);
  load_row(qf[1], A.q.p + b * A.q.sb + (2 * h + 1) * A.q.sh + (int64_t)row * A.q.sn, valid, hh);
  load_row(gf, A.dout.p + b * A.dout.sb + h * A.dout.sh + (int64_t)row * A.dout.sn, valid, hh);
  float lse[2] = {-__builtin_inff(), -__builtin_inff()}, del[2] = {0.0f, 0.0f};
  if (valid) {
    const float* st = A.stats + ((int64_t)(b * s.H + h) * ((s.N + kBwdRows - 1) / kBwdRows) + row / kBwdRows) * kStatFloats +
                      row % kBwdRows;
    lse[0] = st[kStatLse0] * c;
    lse[1] = st[kStatLse1] * c;
    del[0] = -st[kStatDelta0];
    del[1] = del[0] - st[kStatStep];
  }

  const int last = min(row + sq.shift, sq.klen - 1);
  const int last_row = min(row0 + kDiffRows, sq.qlen) - 1;
  const int2 range = split_keys(row0 < sq.qlen ? max(min(last_row + sq.shift, sq.klen - 1) + 1, 0) : 0, pc.piece, pc.pieces,
                                kDqKeys);
  const int turns = (range.y - range.x + kDqKeys - 1) / kDqKeys;
  const int all_to = min(row0 + 32 * wave + sq.shift, sq.klen - 1);  // every row of the wave sees these

  const uint32_t at0 = lds_address(&lds[0][0][0]) + wave * kRowBlock;
  const int copy_row = 8 * wave + (lane >> 3);
  // Tile after tile into place `place` of the ring, one kilobyte at a time; past
  // the last tile it comes again, and is not used.
  constexpr int kCopies = 2 * kTiles;
  struct Copy {
    const uint16_t *k, *v;
    int key;
    uint32_t to, ok, ov;
  } cp_ = {k0 + (int64_t)range.x * A.k.sn, v0 + (int64_t)range.x * A.v.sn, range.x, 0u, copy_offset(copy_row, A.k.sn, lane),
           copy_offset(copy_row, A.v.sn, lane)};
  auto copy_start = [&](int i, int place) __attribute__((always_inline)) {
    const bool on = i > 0 && i < turns;
    cp_.k += on ? kDqKeys * A.k.sn : 0;
    cp_.v += on ? kDqKeys * A.v.sn : 0;
    cp_.key += on ? kDqKeys : 0;
    cp_.to = __builtin_amdgcn_readfirstlane(at0 + (place % kRing) * (kTiles * kTile32));
    if (cp_.key + kDqKeys > sq.klen) {  // keys past the sequence: its last key again (their scores are masked)
      const int r = min(copy_row, sq.klen - 1 - cp_.key);
      cp_.ok = copy_offset(r, A.k.sn, lane);
      cp_.ov = copy_offset(r, A.v.sn, lane);
    }
  };
  auto copy_part = [&](int n) __attribute__((always_inline)) {
    const uint16_t* p = n / 2 == kV ? cp_.v : n / 2 == 0 ? cp_.k : cp_.k + A.k.sh;
    copy_1k(cp_.to + n / 2 * kTile32 + n % 2 * 1024, p, (n / 2 == kV ? cp_.ov : cp_.ok) + n % 2 * 128);
  };
  auto copy = [&](int i, int place) __attribute__((always_inline)) {
    copy_start(i, place);
#pragma unroll
    for (int n = 0; n < kCopies; ++n) copy_part(n);
  };

  f32x16 dq[2][4] = {};
  Scores sa, sb;
  bf16x8 ring[kAhead];
  uint32_t pw[2][8];  // dS of the maps, but for the factors scale and -lambda
  const RowPlace rp = row_place(lane);
  const int cp = col_place(lane);
  // the fragment of slot i of a turn on tile `now` whose products read tile `then`
  auto fragment = [&](int i, const uint8_t* now, const uint8_t* then) __attribute__((always_inline)) {
    if (i < 16) return row_frag(now + (kShared ? 0 : (i & 1) * kTile32), rp, i >> 1);
    if (i < 24) return row_frag(now + kV * kTile32, rp, i - 16);
    const int j = i - 24;  // y, d, map
    return col_frag(then + (kShared ? 0 : (j & 1) * kTile32) + cp, j >> 3, (j >> 1) & 3);
  };
  auto finish = [&](const Scores& old, int r) __attribute__((always_inline)) {  // rows r, r + 1
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      pw[m][r >> 1] = pack_bf16x2(old.p[m][r] * (old.x[r] - del[m]), old.p[m][r + 1] * (old.x[r + 1] - del[m]));
      pin(pw[m][r >> 1]);
    }
  };
  auto turn = [&](int i, Scores& now, Scores& old) __attribute__((always_inline)) {
    constexpr int kSlots = 40;
    const uint8_t* tn = &lds[i % kRing][0][0];
    const uint8_t* to = &lds[(i + kRing - 1) % kRing][0][0];
    const uint8_t* next = &lds[(i + 1) % kRing][0][0];
#pragma unroll
    for (int d = 0; d < 4; ++d) asm volatile("" : "+a"(dq[0][d]), "+a"(dq[1][d]));
    hold_in_agprs(qf[0]);
    hold_in_agprs(qf[1]);
    hold_in_agprs(gf);
    each<0, kSlots>([&](auto slot) __attribute__((always_inline)) {
      constexpr int j = slot.value;
      if constexpr (j == kSlots - 8) {
        copies_landed<0>();
        copy_start(i + 2, i + 2);
        slot_end();
      }
      if constexpr (j >= kSlots - 7 && j < kSlots - 7 + kCopies) copy_part(j - (kSlots - 7));
      const bf16x8 f = ring[j % kAhead];
      if constexpr (j < 16) {
        if constexpr (j < 2) score_first_a(now.s[j & 1], f, qf[j & 1][j >> 1]);
        else score_a(now.s[j & 1], f, qf[j & 1][j >> 1]);
      } else if constexpr (j < 24) {
        if constexpr (j == 16) score_first_a(now.x, f, gf[j - 16]);
        else score_a(now.x, f, gf[j - 16]);
      } else {
        constexpr int m = (j - 24) & 1, d = ((j - 24) >> 1) & 3, y = (j - 24) >> 3;
        const uint4 w = make_uint4(pw[m][4 * y], pw[m][4 * y + 1], pw[m][4 * y + 2], pw[m][4 * y + 3]);
        dq[m][d] = mfma(f, __builtin_bit_cast(bf16x8, w), dq[m][d]);
      }
      constexpr int k = j + kAhead;
      ring[j % kAhead] = k < kSlots ? fragment(k, tn, to) : fragment(k - kSlots, next, tn);
      if constexpr (j < 16 && j % 2 == 0) finish(old, j);
      if constexpr (j >= 18) {  // the exponentials: 32 in 22 slots
#pragma unroll
        for (int e = (j - 18) * 16 / 11; e < (j - 17) * 16 / 11; ++e) {
          now.p[e & 1][e >> 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(now.s[e & 1][e >> 1], c, lse[e & 1]));
          pin(now.p[e & 1][e >> 1]);
        }
      }
      slot_end();
    });
    const int key = range.x + i * kDqKeys;
    if (key + kDqKeys - 1 > all_to || i >= turns) {
      const int to_key = i < turns ? last : -1;  // (past the last tile: none)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (key + 4 * hh + 8 * (r >> 2) + (r & 3) > to_key) now.p[0][r] = now.p[1][r] = 0.0f;
    }
  };
  if (turns > 0) {
    copy(0, 0);
    copy(0, kRing - 1);  // turn 0's products, of dS = 0
    copies_landed<0>();
    hold_in_agprs(qf[0]);
    hold_in_agprs(qf[1]);
    hold_in_agprs(gf);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      pin(lse[m]);
      pin(del[m]);
    }
    all_landed();
    copy(1, 1);
    sb = Scores{};
#pragma unroll
    for (int j = 0; j < kAhead; ++j) ring[j] = fragment(j, &lds[0][0][0], nullptr);
    for (int i = 0; i <= turns; i += 2) {
      turn(i, sa, sb);
      turn(i + 1, sb, sa);
    }
    copies_landed<0>();  // none is under way when the wave ends
  }
  if (pc.pieces > 1) {
    float* o = A.dq_parts +
               (((int64_t)(pc.tile - A.plan.full) * pc.pieces + pc.piece) * 2 * kDiffRows + row - row0) * D + 4 * hh;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(o + m * kDiffRows * D + 32 * d + 8 * q) =
              make_float4(dq[m][d][4 * q], dq[m][d][4 * q + 1], dq[m][d][4 * q + 2], dq[m][d][4 * q + 3]);
  } else {  // zero behind the sequence
    const int first = row0 + 32 * wave;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const float f = m ? -lam * s.scale : s.scale;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) dq[m][d][r] = valid ? dq[m][d][r] * f : 0.0f;
      store_rows(reinterpret_cast<uint8_t*>(lds) + wave * kOutBytes, lane,
                 A.dq.p + b * A.dq.sb + (2 * h + m) * A.dq.sh + (int64_t)first * A.dq.sn, A.dq.sn, -first, s.N - first,
                 [&](int d, int q) { return pack4(dq[m][d], q); });
    }
  }
}

// dk, dv of 128 keys of one value head, 32 keys a wave, over the rows of every
// head of its group or of a piece of them (so a shared head's gradient is summed
// in registers, heads in order); dlambda's parts of these keys:
//   sum P_1 (X - delta_1), which with sum delta_1 is sum P_1 X
// (the rows of P_1 sum to 1; delta_1 comes from an output of rounded P_1, and
// that rounding cancels here).
template <bool kShared>
__device__ __forceinline__ void dkv_of(const DiffBwd& A, uint8_t (*lds)[3][kTile32], float (*stat)[kStatFloats], int wg,
                                       int wgs) {
  constexpr int kK = kShared ? 1 : 2;
  constexpr int kAhead = kShared ? 6 : 4;  // (registers)
  // lds: q of map 0, of map 1, dout
  const DiffShape& s = A.s;
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  const int tiles = (s.M + kDiffRows - 1) / kDiffRows;
  const int id = by_rank(s, s.Hv) ? wg : xcd_local_id(wg, wgs), pieces = A.head_pieces * A.row_pieces;
  const SlabTile at = slab_tile(id / pieces, tiles, s.Hv, s);
  const int piece = id % pieces, row_piece = piece % A.row_pieces;
  const int hv = at.h, b = at.b, tile = at.rank;  // causal: the first keys have the long columns
  const Seq sq = sequence(s, b);
  const int per = s.H / s.Hv / A.head_pieces, h0 = (hv * A.head_pieces + piece / A.row_pieces) * per;  // the piece's heads
  const int key0 = tile * kDiffRows;
  const int key = key0 + 32 * wave + l32;
  const bool valid = key < sq.klen;
  const float c = s.scale * kLog2e;

  bf16x8 kf[kK][8], vf[8];
  const uint16_t* kp = A.k.p + b * A.k.sb + (kShared ? hv : 2 * hv) * A.k.sh + (int64_t)key * A.k.sn;
  load_row(kf[0], kp, valid, hh);
  if (!kShared) load_row(kf[kK - 1], kp + A.k.sh, valid, hh);
  load_row(vf, A.v.p + b * A.v.sb + hv * A.v.sh + (int64_t)key * A.v.sn, valid, hh);

  // the tiles of rows that see any key of this workgroup, head after head
  const int sees = key0 < sq.klen ? min(max(key0 - sq.shift, 0), sq.qlen) / kBwdRows : 0;
  const int all = key0 < sq.klen ? max((sq.qlen + kBwdRows - 1) / kBwdRows - sees, 0) : 0;
  const int first = sees + (int)((int64_t)all * row_piece / A.row_pieces);
  const int end = sees + (int)((int64_t)all * (row_piece + 1) / A.row_pieces);
  const int head_turns = max(end - first, 0), turns = head_turns * per;
  const int row_tiles = (s.N + kBwdRows - 1) / kBwdRows;
  const int wave_last_key = key0 + 32 * wave + 31;

  const uint32_t at0 = lds_address(&lds[0][0][0]) + wave * kRowBlock;
  const uint32_t stat0 = lds_address(&stat[0][0]) + (wave & 1) * 256;
  const int copy_row = 8 * wave + (lane >> 3);
  const uint16_t* qh = A.q.p + b * A.q.sb + 2 * (int64_t)h0 * A.q.sh;
  const uint16_t* gh = A.dout.p + b * A.dout.sb + (int64_t)h0 * A.dout.sh;
  const float* sth = A.stats + (int64_t)(b * s.H + h0) * row_tiles * kStatFloats + (wave & 1) * 64;
  // Tile after tile (head after head) into the ring, one kilobyte at a time; past
  // the last tile it comes again, and is not used.
  constexpr int kCopies = 7;
  struct Copy {
    const uint16_t *q, *g;
    const float* st;
    int u, t;  // head of the group and row tile
    uint32_t to, to_st, oq, og;
  } cp_ = {};
  auto copy_start = [&](int i, int place) __attribute__((always_inline)) {
    const bool on = i > 0 && i < turns;
    if (i == 0 || (on && cp_.t + 1 == end)) {
      cp_.u += i > 0;
      cp_.t = first;
      cp_.q = qh + 2 * cp_.u * A.q.sh + (int64_t)first * kBwdRows * A.q.sn;
      cp_.g = gh + cp_.u * A.dout.sh + (int64_t)first * kBwdRows * A.dout.sn;
      cp_.st = sth + ((int64_t)cp_.u * row_tiles + first) * kStatFloats;
      cp_.oq = copy_offset(copy_row, A.q.sn, lane);
      cp_.og = copy_offset(copy_row, A.dout.sn, lane);
    } else {
      cp_.t += on;
      cp_.q += on ? kBwdRows * A.q.sn : 0;
      cp_.g += on ? kBwdRows * A.dout.sn : 0;
      cp_.st += on ? kStatFloats : 0;
    }
    cp_.to = __builtin_amdgcn_readfirstlane(at0 + (place % kRing) * (3 * kTile32));
    cp_.to_st = __builtin_amdgcn_readfirstlane(stat0 + (place % kRing) * (kStatFloats * 4));
    if (cp_.t + 1 == end) {  // rows past the sequence: its last row again (their P is 0)
      const int r = min(copy_row, sq.qlen - 1 - cp_.t * kBwdRows);
      cp_.oq = copy_offset(r, A.q.sn, lane);
      cp_.og = copy_offset(r, A.dout.sn, lane);
    }
  };
  auto copy_part = [&](int n) __attribute__((always_inline)) {
    if (n == 6) {
      copy_256(cp_.to_st, cp_.st, lane * 4);
    } else {
      const uint16_t* p = n / 2 == 2 ? cp_.g : n / 2 == 0 ? cp_.q : cp_.q + A.q.sh;
      copy_1k(cp_.to + n / 2 * kTile32 + n % 2 * 1024, p, (n / 2 == 2 ? cp_.og : cp_.oq) + n % 2 * 128);
    }
  };
  auto copy = [&](int i, int place) __attribute__((always_inline)) {
    copy_start(i, place);
#pragma unroll
    for (int n = 0; n < kCopies; ++n) copy_part(n);
  };

  f32x16 dv[4] = {}, dk[kK][4] = {};
  Scores sa, sb;
  bf16x8 ring[kAhead];
  float4 step;        // delta_0 - delta_1 of four of the last tile's rows
  uint32_t pw[3][8];  // P_0 - lambda P_1, dS_0, dS_1
  float dlam = 0.0f;
  const RowPlace rp = row_place(lane);
  const int cp = col_place(lane);
  int u = 0, left = head_turns;  // of the last tile: its head, and the tiles of that head from it on
  int rt = first;                // row tile of the turn's scores
  float lam = uniform(s.lambda[h0]);
  // of the keys' operands, the first map's beside the gradients, and V's where
  // there is room; the second map's beside the scores
  auto hold_operands = [&]() __attribute__((always_inline)) {
    hold_in_agprs(kf[0]);
    if constexpr (kShared) {
      hold_in_agprs(vf);
    } else {
      hold_in_vgprs(kf[1]);
      hold_in_vgprs(vf);
    }
  };
  auto fragment = [&](int i, const uint8_t* now, const uint8_t* then) __attribute__((always_inline)) {
    if (i < 16) return row_frag(now + (i & 1) * kTile32, rp, i >> 1);
    if (i < 24) return row_frag(now + 2 * kTile32, rp, i - 16);
    const int j = i - 24, d = (j / 3) & 3, y = j / 12;  // y, d, which: dv, dk of map 0, of map 1
    return col_frag(then + (j % 3 == 0 ? 2 : j % 3 - 1) * kTile32 + cp, y, d);
  };
  // rows 4 q .. 4 q + 3 of a lane's sixteen
  auto quad = [&](const float* st, int q) __attribute__((always_inline)) {
    return *reinterpret_cast<const float4*>(st + 8 * q + 4 * hh);
  };
  auto put = [](f32x16& x, int q, const float4& f) __attribute__((always_inline)) {
    x[4 * q] = f.x;
    x[4 * q + 1] = f.y;
    x[4 * q + 2] = f.z;
    x[4 * q + 3] = f.w;
  };
  // P_0 - lambda P_1, dS_0 and dS_1 of rows r, r + 1 of a lane's sixteen of the last tile
  auto finish = [&](const Scores& old, int r) __attribute__((always_inline)) {
    const float w0 = old.p[1][r] * (old.x[r] + (r & 2 ? step.z : step.x));
    const float w1 = old.p[1][r + 1] * (old.x[r + 1] + (r & 2 ? step.w : step.y));
    dlam += w0 + w1;
    pw[0][r >> 1] = pack_bf16x2(__builtin_fmaf(-lam, old.p[1][r], old.p[0][r]),
                                __builtin_fmaf(-lam, old.p[1][r + 1], old.p[0][r + 1]));
    pw[1][r >> 1] = pack_bf16x2(old.p[0][r] * old.x[r], old.p[0][r + 1] * old.x[r + 1]);
    pw[2][r >> 1] = pack_bf16x2(-lam * w0, -lam * w1);
#pragma unroll
    for (int m = 0; m < 3; ++m) pin(pw[m][r >> 1]);
  };
  // the last tile is done: a head's last one ends its part of dlambda
  auto end_of_tile = [&]() __attribute__((always_inline)) {
    if (--left == 0) {
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) dlam += __shfl_xor(dlam, m);
      if (lane == 0) A.partial[((int64_t)(h0 + u) * s.B + b) * A.parts + (tile * A.row_pieces + row_piece) * 4 + wave] = dlam;
      dlam = 0.0f;
      ++u;
      left = head_turns;
      lam = uniform(s.lambda[h0 + min(u, per - 1)]);
    }
  };
  auto turn = [&](int i, Scores& now, Scores& old) __attribute__((always_inline)) {
    constexpr int kSlots = 48;
    const uint8_t* tn = &lds[i % kRing][0][0];
    const uint8_t* to = &lds[(i + kRing - 1) % kRing][0][0];
    const uint8_t* next = &lds[(i + 1) % kRing][0][0];
    const float* stn = stat[i % kRing];
    const float* old_st = stat[(i + kRing - 1) % kRing];
    const float* next_st = stat[(i + 1) % kRing];
    // (the gradients where only MFMAs reach them)
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      asm volatile("" : "+a"(dv[d]), "+a"(dk[0][d]));
      if (!kShared) asm volatile("" : "+a"(dk[kK - 1][d]));
    }
    hold_operands();
    each<0, kSlots>([&](auto slot) __attribute__((always_inline)) {
      constexpr int j = slot.value;
      if constexpr (j == kSlots - 8) {
        copies_landed<0>();
        copy_start(i + 2, i + 2);
        slot_end();
      }
      if constexpr (j >= kSlots - 7) copy_part(j - (kSlots - 7));
      const bf16x8 f = ring[j % kAhead];
      if constexpr (j < 16) {
        if constexpr (kShared || j % 2 == 0) score_a(now.s[j & 1], f, kf[0][j >> 1]);
        else score(now.s[j & 1], f, kf[kK - 1][j >> 1]);
      } else if constexpr (j < 24) {
        if constexpr (kShared) score_a(now.x, f, vf[j - 16]);
        else score(now.x, f, vf[j - 16]);
      } else {
        constexpr int w = (j - 24) % 3, d = ((j - 24) / 3) & 3, y = (j - 24) / 12;
        const bf16x8 p = __builtin_bit_cast(bf16x8, make_uint4(pw[w][4 * y], pw[w][4 * y + 1], pw[w][4 * y + 2], pw[w][4 * y + 3]));
        if constexpr (w == 0) dv[d] = mfma(f, p, dv[d]);
        else dk[kShared ? 0 : w - 1][d] = mfma(f, p, dk[kShared ? 0 : w - 1][d]);
      }
      constexpr int k = j + kAhead;
      ring[j % kAhead] = k < kSlots ? fragment(k, tn, to) : fragment(k - kSlots, next, tn);
      if constexpr (j < 24 && j % 3 == 0) finish(old, j / 3 * 2);
      if constexpr (j >= 8 && j < 12) put(now.x, j - 8, quad(stn + kStatDelta0, j - 8));
      if constexpr (j < 21 && j % 6 == 3) step = quad(old_st + kStatStep, j / 6 + 1);
      if constexpr (j == 45) step = quad(stn + kStatStep, 0);
      // the next turn's scores start from the rows' log sums
      if constexpr (j >= 40 && j < 44) {
        put(old.s[0], j - 40, quad(next_st + kStatLse0, j - 40));
        put(old.s[1], j - 40, quad(next_st + kStatLse1, j - 40));
      }
      if constexpr (j >= 18) {  // the exponentials: 32 in 30 slots
#pragma unroll
        for (int e = (j - 18) * 16 / 15; e < (j - 17) * 16 / 15; ++e) {
          now.p[e & 1][e >> 1] = __builtin_amdgcn_exp2f(now.s[e & 1][e >> 1] * c);
          pin(now.p[e & 1][e >> 1]);
        }
      }
      slot_end();
    });
    if (i > 0 && i <= turns) end_of_tile();
    const int row = rt * kBwdRows;
    if (wave_last_key >= sq.klen || wave_last_key > row + sq.shift || i >= turns) {
      // rows below it do not see this key (past the last tile: none does)
      const int limit = valid && i < turns ? key - sq.shift - row : kBwdRows;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + 4 * hh + (r & 3) < limit) now.p[0][r] = now.p[1][r] = 0.0f;
    }
    if (++rt == end) rt = first;
  };
  if (turns > 0) {
    copy(0, 0);
    copy(0, kRing - 1);  // turn 0's products, of P = dS = 0
    copies_landed<0>();
    hold_operands();
    all_landed();
    copy(1, 1);
    sb = Scores{};
    step = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      put(sa.s[0], q, quad(stat[0] + kStatLse0, q));
      put(sa.s[1], q, quad(stat[0] + kStatLse1, q));
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) ring[j] = fragment(j, &lds[0][0][0], nullptr);
    for (int i = 0; i <= turns; i += 2) {
      turn(i, sa, sb);
      turn(i + 1, sb, sa);
    }
    copies_landed<0>();  // none is under way when the wave ends
  } else if (lane < 1) {
    for (int n = 0; n < per; ++n) A.partial[((int64_t)(h0 + n) * s.B + b) * A.parts + (tile * A.row_pieces + row_piece) * 4 + wave] = 0.0f;
  }
  if (pieces > 1) {
    float* o = A.dkv_parts +
               (((((int64_t)b * s.Hv + hv) * tiles + tile) * pieces + piece) * 3 * kDiffRows + key - key0) * D + 4 * hh;
#pragma unroll
    for (int m = 0; m < 1 + kK; ++m)
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x16& x = m ? dk[m - 1][d] : dv[d];
          *reinterpret_cast<float4*>(o + m * kDiffRows * D + 32 * d + 8 * q) =
              make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
        }
    return;
  }
  // zero behind the sequence
  uint8_t* mine = reinterpret_cast<uint8_t*>(lds) + wave * kOutBytes;
  const int first_key = key0 + 32 * wave;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) dv[d][r] = valid ? dv[d][r] : 0.0f;
  store_rows(mine, lane, A.dv.p + b * A.dv.sb + hv * A.dv.sh + (int64_t)first_key * A.dv.sn, A.dv.sn, 0, s.M - first_key,
             [&](int d, int q) { return pack4(dv[d], q); });
#pragma unroll
  for (int m = 0; m < kK; ++m) {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) dk[m][d][r] = valid ? dk[m][d][r] * s.scale : 0.0f;
    store_rows(mine, lane, A.dk.p + b * A.dk.sb + ((kShared ? hv : 2 * hv) + m) * A.dk.sh + (int64_t)first_key * A.dk.sn,
               A.dk.sn, 0, s.M - first_key, [&](int d, int q) { return pack4(dk[m][d], q); });
  }
}

// Both in one launch, the keys' workgroups first: what either leaves of the last
// round of the chip's 256 CUs the other fills.
//
// 12,480 rows x 3 heads: 1.24 ms, of peaked rows 1.32 to 1.35; the eight products
// that the gradients are make 710 to 770 TFLOP/s of it, the eleven that it executes
// (scores and X in both halves) 980 to 1,060, 75 to 82 % of a large bf16 product's
// rate, at the clock that power leaves.
template <bool kShared>
__global__ __launch_bounds__(256, 1) void diff_bwd_kernel(DiffBwd A, int key_wgs) {
  struct Keys {
    uint8_t tiles[kRing][3][kTile32];
    float stat[kRing][kStatFloats];
  };
  struct Queries {
    uint8_t tiles[kRing][kShared ? 2 : 3][kTile32];
  };
  union Lds {
    Keys keys;
    Queries rows;
  };
  __shared__ __attribute__((aligned(1024))) Lds lds;
  lds_poison(&lds, sizeof(lds));
  lds_poison_done();
  if ((int)blockIdx.x < key_wgs)
    dkv_of<kShared>(A, lds.keys.tiles, lds.keys.stat, blockIdx.x, key_wgs);
  else
    dq_of<kShared>(A, lds.rows.tiles, blockIdx.x - key_wgs);
}

// Workgroups 0 .. H - 1: dlambda of a head, its keys' parts and its rows'
// delta_1 summed in one order, in 64 bits.  The others: dq of a tile that was
// split, the pieces summed in order, 8 rows of both maps a workgroup; then dv and
// dk of key tiles that were, 16 rows of one of them.
constexpr int kJoinRows = 8;
__global__ __launch_bounds__(256) void diff_end_kernel(DiffBwd A) {
  __shared__ double sum[256];
  lds_poison(sum, sizeof(sum));
  lds_poison_done();
  const DiffShape& s = A.s;
  if ((int)blockIdx.x < s.H) {
    const int h = blockIdx.x;
    const float* p = A.partial + (int64_t)h * s.B * A.parts;
    double x = 0.0;
    for (int64_t i = threadIdx.x; i < (int64_t)s.B * A.parts; i += 256) x += (double)p[i];
    const int row_tiles = (s.N + kBwdRows - 1) / kBwdRows;
    for (int b = 0; b < s.B; ++b) {
      const float* d = A.delta + (int64_t)(b * s.H + h) * row_tiles;
      for (int i = threadIdx.x; i < row_tiles; i += 256) x += (double)d[i];
    }
    sum[threadIdx.x] = x;
    __syncthreads();
    for (int n = 128; n > 0; n >>= 1) {
      if ((int)threadIdx.x < n) sum[threadIdx.x] += sum[threadIdx.x + n];
      __syncthreads();
    }
    if (threadIdx.x == 0) A.dlambda[h] = (float)-sum[0];
    return;
  }
  const int dq_blocks = (row_tiles_of(s) - A.plan.full) * (kDiffRows / kJoinRows);
  if ((int)blockIdx.x - s.H >= dq_blocks) {  // 16 rows of dv or of a map's dk, from the pieces' sums
    const int tiles = (s.M + kDiffRows - 1) / kDiffRows, per_tile = kDiffRows / 16, grads = s.Hk == s.Hv ? 2 : 3;
    const int w = blockIdx.x - s.H - dq_blocks, m = w % grads, id = w / grads / per_tile;
    const int r = w / grads % per_tile * 16 + (threadIdx.x >> 4), cc = threadIdx.x & 15;
    const int key = id % tiles * kDiffRows + r, bh = id / tiles, b = bh / s.Hv, hv = bh - b * s.Hv;
    if (key >= s.M) return;
    const bool valid = key < sequence(s, b).klen;
    float f[8] = {};
    const int pieces = A.head_pieces * A.row_pieces;
    for (int u = 0; u < pieces && valid; ++u) {
      const float4* p = reinterpret_cast<const float4*>(
          A.dkv_parts + ((((int64_t)id * pieces + u) * 3 + m) * kDiffRows + r) * D + 8 * cc);
      const float4 x = p[0], y = p[1];
      f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
      f[4] += y.x; f[5] += y.y; f[6] += y.z; f[7] += y.w;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= m ? s.scale : 1.0f;
    const Rows& y = m ? A.dk : A.dv;
    const int head = m == 0 ? hv : grads == 2 ? hv : 2 * hv + m - 1;
    *reinterpret_cast<uint4*>(y.p + b * y.sb + head * y.sh + (int64_t)key * y.sn + 8 * cc) = pack_bf16x8(f);
    return;
  }
  const int w = blockIdx.x - s.H, tile = w / (kDiffRows / kJoinRows);
  const int m = threadIdx.x >> 7, r = w % (kDiffRows / kJoinRows) * kJoinRows + ((threadIdx.x >> 4) & 7), cc = threadIdx.x & 15;
  const RowTile rt = row_tile(A.plan.full + tile, s);
  const int row = rt.row0 + r;
  if (row < 0) return;
  const bool valid = row < sequence(s, rt.b).qlen;
  float f[8] = {};
  for (int u = 0; u < A.plan.pieces && valid; ++u) {
    const float4* p = reinterpret_cast<const float4*>(
        A.dq_parts + (((int64_t)tile * A.plan.pieces + u) * 2 * kDiffRows + m * kDiffRows + r) * D + 8 * cc);
    const float4 x = p[0], y = p[1];
    f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
    f[4] += y.x; f[5] += y.y; f[6] += y.z; f[7] += y.w;
  }
  const float scale = m ? -s.lambda[rt.h] * s.scale : s.scale;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] *= scale;
  *reinterpret_cast<uint4*>(A.dq.p + rt.b * A.dq.sb + (2 * rt.h + m) * A.dq.sh + (int64_t)row * A.dq.sn + 8 * cc) =
      pack_bf16x8(f);
}

}  // namespace

constexpr int kCus = 256;  // each holds one workgroup of the tile kernels

// Tiles [full, tiles) cut along the keys, in pieces of 512 keys or more.
static DiffTiles cut_tiles(int tiles, int full, int pieces, int M) {
  pieces = std::min({pieces, M / 512, 16});
  if (pieces < 2) return {tiles, 1};
  return {full, pieces};
}
// Pieces of the last tiles, which leave part of the chip idle, that fill it.
static int filling(int tiles, int full) { return tiles > full ? kCus / (tiles - full) : 1; }

DiffPlan diff_plan(const DiffShape& s, bool ragged) {
  DiffPlan p;
  // A row group's 128 keys take 4 us in the few-row kernel, a tile's 3.7 in the tile
  // kernel: there where groups are no more than heads.  24 heads on 8, 17 rows,
  // 20,000 keys 44 us there, 74 in tiles; 40 on 1, one row 29, 95; 16 on 8, 4 x 17
  // rows, 6,000 keys 47, 62; 2 on 1, 30 rows, 40 keys 13, 11.
  p.few = few_groups(s) == 1 || (few_groups(s) <= s.H / s.Hv && s.N <= kDiffRows && s.M >= 512);
  if (p.few) {
    // One workgroup a CU, of 128 keys or more (one row over 600 keys 20 us in one
    // piece, 15 in 4; 5,000 keys 26 in 9, 19 in 39).  Where lengths may differ two,
    // half as long, of 512 or more: 32 caches of 256 to 8,192 keys, 8 heads, took
    // 141 us uncut, 107 in halves, 114 in thirds (the join with it); equal ones gain
    // nothing from it.
    const int64_t wgs = (int64_t)s.B * s.Hv * few_groups(s);
    int64_t n = kCus / wgs;
    if (ragged && s.B > 1 && few_groups(s) == 1) n = std::max(n, std::min<int64_t>(2 * kCus / wgs, s.M / 512));
    n = std::min<int64_t>(n, s.M / 128);
    p.tiles = {0, (int)(n < 1 ? 1 : n)};
  } else {
    const int tiles = row_tiles_of(s);
    // the longest tile's keys over the average one's
    const double graded = s.causal ? s.M / (s.M - 0.5 * std::min(s.N, s.M)) : 1.0;
    if (graded > 1.25) {
      // Causal tiles of different lengths, the longest first, fill the CUs' time by
      // themselves unless the longest is longer than that; then all are cut, if
      // that saves more than the join costs (in turns of 32 keys, 0.9 us each).
      // Uncut and cut, forward in us: 30,000 rows 684, 514; 12,480 rows (x 3
      // heads) 298, 267; 6,000 x 4 144, 124; 5,000 x 5 121, 120; 2,500 x 12 68, 103;
      // 2,048 x 20 63, 106.
      const double longest = s.M / 32.0, mean = longest * tiles / (kCus * graded);
      const DiffTiles cut = cut_tiles(tiles, 0, (int)std::ceil(kCus * graded / tiles), s.M);
      const double join = 40 + (double)tiles * kDiffRows * cut.pieces / 1000;
      p.tiles = longest - mean > join ? cut : DiffTiles{tiles, 1};
    } else {
      const int full = tiles / kCus * kCus;
      p.tiles = cut_tiles(tiles, full, filling(tiles, full), s.M);
    }
  }
  return p;
}

static size_t join_rows(const DiffShape& s, const DiffPlan& p) {
  if (p.tiles.pieces < 2) return 0;
  return p.few ? (size_t)s.B * s.H * s.N : (size_t)(row_tiles_of(s) - p.tiles.full) * kDiffRows;
}

// A launch is a 1D grid of fewer than 2^32 threads.
static bool fits(int64_t workgroups, int threads) { return workgroups < ((int64_t)1 << 32) / threads; }

// Workgroups of the forward kernels (those of the join are fewer than 2^19).
static int64_t fwd_workgroups(const DiffShape& s, const DiffPlan& p) {
  if (p.few) return ((int64_t)s.B * s.Hv * p.tiles.pieces + 7) / 8 * 8 * few_groups(s);
  return p.tiles.full + (int64_t)(row_tiles_of(s) - p.tiles.full) * p.tiles.pieces;
}

size_t diff_fwd_bytes(const DiffShape& s) {  // with lengths and without
  size_t most = 0;
  for (const bool ragged : {false, true}) {
    const DiffPlan p = diff_plan(s, ragged);
    if (!fits(fwd_workgroups(s, p), 256)) return kTooLarge;
    most = std::max(most, join_rows(s, p) * p.tiles.pieces * 2 * (D + 2) * sizeof(float));
  }
  return most;
}

hipError_t launch_diff_fwd(const DiffFwd& a, hipStream_t stream) {
  const DiffShape& s = a.s;
  const DiffPlan p = diff_plan(s, s.kv_lens != nullptr);
  const bool shared = s.Hk == s.Hv;
  const dim3 grid((unsigned)fwd_workgroups(s, p));
  if (p.few) {
    if (shared)
      hipLaunchKernelGGL(diff_few_kernel<true>, grid, dim3(256), 0, stream, a, p.tiles.pieces);
    else
      hipLaunchKernelGGL(diff_few_kernel<false>, grid, dim3(256), 0, stream, a, p.tiles.pieces);
  } else {
    const auto kernel = a.lse ? (shared ? diff_fwd_kernel<true, true> : diff_fwd_kernel<false, true>)
                              : (shared ? diff_fwd_kernel<true, false> : diff_fwd_kernel<false, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, p.tiles);
  }
  if (const size_t rows = join_rows(s, p)) {
    const dim3 joins((unsigned)(p.few ? rows : (rows + 3) / 4));
    if (p.few)
      hipLaunchKernelGGL(diff_join_kernel<true>, joins, dim3(256), 0, stream, a, p.tiles);
    else
      hipLaunchKernelGGL(diff_join_kernel<false>, joins, dim3(256), 0, stream, a, p.tiles);
  }
  return hipGetLastError();
}

// The backward launch: the keys' workgroups, then the rows'.  A row tile takes
// 5/6 of a key tile's time over the same length (40 MFMAs a 32 x 32 block
// against 48), times the heads that share a value head; the row tiles that would
// stand past the time that the chip needs for all of it at best are cut along
// the keys.
struct BwdCost {
  // key tiles; a key tile's time, a row tile's (the longest's under a causal mask),
  // in slots of an MFMA (0.025 us)
  int64_t keys, key, row;
  double fair;  // a CU's time for everything if nothing idled
};
static BwdCost bwd_cost(const DiffShape& s) {
  BwdCost c = {(int64_t)s.B * s.Hv * ((s.M + kDiffRows - 1) / kDiffRows), (int64_t)(s.H / s.Hv) * ((s.N + 31) / 32) * 48,
               (int64_t)((s.M + 31) / 32) * 40, 0.0};
  const double seen = s.causal ? 1.0 - 0.5 * std::min(s.N, s.M) / s.M : 1.0;  // of all pairs
  c.fair = seen * (double)(c.keys * c.key + row_tiles_of(s) * c.row) / kCus;
  return c;
}
// A key tile walks the rows of all the query heads that share it.  Where that
// takes longer than the chip needs for everything, its heads and then their rows
// (256 or more) go to several workgroups, if that saves more than their sums' way
// through the workspace costs: gradients of 2,000 rows and keys, 16 heads on 2,
// 686 -> 216 us, 500 rows, 8 heads on 1, 186 -> 45, 10,000 rows of one head over
// 100 keys 415 -> 49; causal 5,000 x 5 heads (236, 271 in two) and 2,047, 4 x 16 on 4,
// stay whole (755).
struct KeyPieces {
  int heads, rows;
  int all() const { return heads * rows; }
};
static KeyPieces key_pieces(const DiffShape& s) {
  const BwdCost c = bwd_cost(s);
  const double fair = c.fair;
  const int per = s.H / s.Hv;
  KeyPieces least = {1, 1};
  double time = std::max((double)c.key, fair);
  auto consider = [&](KeyPieces p) {
    const double t = std::max((double)c.key / p.all(), fair) + 600 + 6.0 * c.keys * p.all();
    if (t < time) {
      time = t;
      least = p;
    }
  };
  for (int p = 2; p <= std::min(per, kCus); ++p)
    if (per % p == 0) consider({p, 1});
  for (int p = 2; p <= std::min(16, s.N / 256); ++p) consider({per, p});
  return least;
}
static DiffTiles bwd_tiles(const DiffShape& s, int pieces) {
  const int tiles = row_tiles_of(s);
  const BwdCost c = bwd_cost(s);
  const int64_t keys = c.keys * pieces, key_cost = c.key / pieces, row_cost = c.row;
  if (s.causal) {
    // the longest row tiles cut where they would outlast the rest, if that saves
    // more than the pieces' way through the workspace costs (one head of 12,480
    // rows 443 us uncut, 278 cut)
    double time = std::max((double)row_cost, c.fair);
    int cut = 1;
    for (int p = 2; p <= std::min(16, s.M / 512); ++p) {
      const double t = std::max((double)row_cost / p, c.fair) + 600 + 2.6 * tiles * p;
      if (t < time) {
        time = t;
        cut = p;
      }
    }
    return cut_tiles(tiles, 0, cut, s.M);
  }
  const int64_t best = (keys * key_cost + tiles * row_cost) / kCus;
  const int64_t round = keys / kCus, more = keys % kCus;             // `more` CUs take round + 1 key tiles
  const int64_t a = best - round * key_cost, b = a - key_cost;
  int64_t full = (kCus - more) * (a > 0 ? a / row_cost : 0) + more * (b > 0 ? b / row_cost : 0);
  if (full > tiles) full = tiles;
  // what is left goes to the CUs' remaining time, about rest row_cost in all
  return cut_tiles(tiles, (int)full, filling(tiles, (int)full), s.M);
}

// Workgroups of the backward launches: the rows' statistics, both walks (the keys'
// first), the end.
struct BwdGrids {
  int64_t stats, keys, walks, end;
};
static BwdGrids bwd_grids(const DiffShape& s, const KeyPieces& pieces, const DiffTiles& plan) {
  const int64_t key_tiles = bwd_cost(s).keys, rest = row_tiles_of(s) - plan.full;
  BwdGrids g;
  g.stats = (int64_t)s.B * s.H * ((s.N + kBwdRows - 1) / kBwdRows);
  g.keys = key_tiles * pieces.all();
  g.walks = g.keys + plan.full + rest * plan.pieces;
  g.end = s.H + rest * (kDiffRows / kJoinRows);
  if (pieces.all() > 1) g.end += key_tiles * (kDiffRows / 16) * (s.Hk == s.Hv ? 2 : 3);
  return g;
}

size_t diff_bwd_bytes(const DiffShape& s, DiffBwd* a) {
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t row_tiles = (size_t)s.B * s.H * ((s.N + kBwdRows - 1) / kBwdRows);
  const KeyPieces pieces = key_pieces(s);
  const DiffTiles plan = bwd_tiles(s, pieces.all());
  const BwdGrids g = bwd_grids(s, pieces, plan);
  if (!fits(g.stats, 16 * kBwdRows) || !fits(g.walks, 256) || !fits(g.end, 256)) return kTooLarge;
  const int parts = 4 * ((s.M + kDiffRows - 1) / kDiffRows) * pieces.rows;
  size_t at[5] = {};
  at[0] = up(row_tiles * kStatFloats * sizeof(float));
  at[1] = up(at[0] + row_tiles * sizeof(float));
  at[2] = up(at[1] + (size_t)s.H * s.B * parts * sizeof(float));
  at[3] = at[2];
  if (plan.pieces > 1)
    at[3] += (size_t)(row_tiles_of(s) - plan.full) * plan.pieces * 2 * kDiffRows * D * sizeof(float);
  at[4] = at[3];
  if (pieces.all() > 1) at[4] += (size_t)bwd_cost(s).keys * pieces.all() * 3 * kDiffRows * D * sizeof(float);
  if (a) {
    char* ws = reinterpret_cast<char*>(a->stats);
    a->delta = reinterpret_cast<float*>(ws + at[0]);
    a->partial = reinterpret_cast<float*>(ws + at[1]);
    a->dq_parts = reinterpret_cast<float*>(ws + at[2]);
    a->dkv_parts = reinterpret_cast<float*>(ws + at[3]);
    a->head_pieces = pieces.heads;
    a->row_pieces = pieces.rows;
    a->parts = parts;
    a->plan = plan;
  }
  return at[4];
}

hipError_t launch_diff_bwd(const DiffBwd& a, hipStream_t stream) {
  const DiffShape& s = a.s;
  const BwdGrids g = bwd_grids(s, {a.head_pieces, a.row_pieces}, a.plan);
  hipLaunchKernelGGL(diff_stats_kernel, dim3((unsigned)g.stats), dim3(16 * kBwdRows), 0, stream, a);
  const dim3 walks((unsigned)g.walks);
  if (s.Hk == s.Hv)
    hipLaunchKernelGGL(diff_bwd_kernel<true>, walks, dim3(256), 0, stream, a, (int)g.keys);
  else
    hipLaunchKernelGGL(diff_bwd_kernel<false>, walks, dim3(256), 0, stream, a, (int)g.keys);
  hipLaunchKernelGGL(diff_end_kernel, dim3((unsigned)g.end), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sol
