// Cross attention (sol_cross_attn_fwd, _bwd): softmax attention of one sequence's
// rows to another's keys and values, of a length of its own,
//   out = softmax(scale q k^T) v over the keys that are visible.
//
// As in the differential attention one pass over the keys with the running maximum
// and sum of each row; scores S^T = K Q^T and outputs O^T = V^T P^T, so that a lane
// owns a row and P as the score MFMA leaves it is the operand of the next.  fp32
// throughout but for the operands: P is rounded to bf16, as the values are bf16, and
// its product divided by the sum of the rounded ones.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "sol_cross.h"
#include "sol_softmax.h"

namespace sol {
namespace {

__device__ __forceinline__ int query_len(const CrossShape& s, int b) {
  return s.q_lens ? min(max(s.q_lens[b], 0), s.N) : s.N;
}
__device__ __forceinline__ int key_len(const CrossShape& s, int b) {
  return s.kv_lens ? min(max(s.kv_lens[b], 0), s.M) : s.M;
}

// Sequence and head of slab `slab`; where lengths differ head after head, so that every
// XCD has some of each sequence.
__device__ __forceinline__ int2 slab_of(int slab, int heads, const CrossShape& s) {  // (b, h)
  return s.q_lens || s.kv_lens || s.mask ? make_int2(slab % s.B, slab / s.B) : make_int2(slab / heads, slab % heads);
}

// Results of pieces of the keys, to be joined: o fp32 [piece][row][128], then the
// log2 of the sums that o was divided by, [piece][row], and of the exact ones (for
// training), for `rows` rows: those of the tiles that are split (tile after tile),
// or, where the few-row kernel splits, all [B][H][N].
struct Parts {
  float *o, *l, *exact;
  int64_t rows;
};
__device__ __forceinline__ Parts parts_of(float* ws, int64_t rows, int pieces) {
  return {ws, ws + rows * pieces * D, ws + rows * pieces * (D + 1), rows};
}

// out, and for training what its rounding left, of two dims from `d` of row (b, h, n).
__device__ __forceinline__ void store_two(const CrossFwd& A, int b, int h, int n, int d, float2 o) {
  const uint32_t w = pack_bf16x2(o.x, o.y);
  *reinterpret_cast<uint32_t*>(A.out.p + b * A.out.sb + h * A.out.sh + (int64_t)n * A.out.sn + d) = w;
  if (A.left)
    *reinterpret_cast<uint32_t*>(A.left + (((int64_t)b * A.s.H + h) * A.s.N + n) * D + d) = left2(o.x, o.y, w);
}

// ------------------------------------------------------------------- forward

// Groups of rows of one key head's query heads in the few-row kernel.
__host__ __device__ inline int64_t few_groups(const CrossShape& s) {
  return ((int64_t)(s.H / s.Hk) * s.N + kFewRows - 1) / kFewRows;
}

// Rows in groups of 32 of all heads that share a key head -- row r is token r % N of
// head hk per + r / N --, a workgroup each: each of its eight waves walks every eighth
// block of 32 keys on its own, through LDS of its own (no barriers), the next block's
// bytes in flight in its registers; the waves' rows are joined at the end.  A key that is
// masked is not read.
constexpr int kFewWaves = 8, kFewThreads = 64 * kFewWaves;
template <bool kMasked>
__global__ __launch_bounds__(kFewThreads) void cross_few_kernel(CrossFwd A, int nsplit) {
  constexpr int kBlock = 32, kWaves = kFewWaves;
  constexpr int kTileElems = kBlock * kStride;
  constexpr int kRow = D + 4;
  struct Joined {
    float o[kWaves][kFewRows][kRow];
    float m[kWaves][kFewRows], l[kWaves][kFewRows], exact[kWaves][kFewRows];
  };
  union Lds {
    uint16_t tiles[kWaves][2 * kTileElems];
    Joined j;
  };
  __shared__ __attribute__((aligned(16))) Lds lds;
  lds_poison(&lds, sizeof(lds));
  lds_poison_done();
  const CrossShape& s = A.s;
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  // (sequence, key head, piece of the keys) after another over the XCDs; where several
  // groups of rows read the same keys they are side by side on one, as many on each XCD
  // (whole heads on an XCD: 20 heads of 11 groups over 901 keys 30 us, so 18; one head of
  // 81 over 1,182 47, 21)
  const int per = s.H / s.Hk, groups = (int)few_groups(s);
  int id = groups > 1 ? xcd_local_id(blockIdx.x, gridDim.x) : blockIdx.x;
  const int64_t row_base = (int64_t)(id % groups) * kFewRows;
  const int n_rows = (int)min((int64_t)per * s.N - row_base, (int64_t)kFewRows);
  id /= groups;
  const int split = id % nsplit;
  id /= nsplit;
  const int2 bh = groups > 1 ? slab_of(id, s.Hk, s) : make_int2(id / s.Hk, id % s.Hk);
  const int hk = bh.y, b = bh.x;
  const int qlen = query_len(s, b), klen = key_len(s, b);
  const float c = s.scale * kLog2e;
  const int64_t my = row_base + min(l32, n_rows - 1);
  const int h = hk * per + (int)(my / s.N), row = (int)(my % s.N);
  const bool valid = l32 < n_rows && row < qlen;

  const uint16_t* k = A.k.p + b * A.k.sb + hk * A.k.sh;
  const uint16_t* v = A.v.p + b * A.v.sb + hk * A.v.sh;
  const uint8_t* mk = kMasked ? s.mask + (int64_t)b * s.M : nullptr;
  bf16x8 qf[8];
  if (!__any(valid)) return;  // (the same in all waves)
  load_row(qf, A.q.p + b * A.q.sb + h * A.q.sh + (int64_t)row * A.q.sn, valid, hh);

  const int2 range = split_keys(klen, split, nsplit, kBlock * kWaves);
  MapRows x;
  clear(x);
  uint16_t* tk = lds.tiles[wave];
  uint16_t* tv = tk + kTileElems;
  const int tr = column_offset(lane);
  // Which keys of a block are visible, a bit each.
  auto seen_byte = [&](int key) __attribute__((always_inline)) {
    const int i = key + l32;
    return kMasked ? (i < range.y ? (int)mk[i] : 0) : (int)(i < range.y);
  };
  auto seen_word = [&](int byte) __attribute__((always_inline)) { return (uint32_t)__ballot(byte != 0); };
  constexpr int kLoads = kBlock / 4;  // rows of a lane's: lane / 16 + 4 u
  uint4 xk[kLoads], xv[kLoads];
  const int lr = lane >> 4, cc = lane & 15;
  auto load = [&](int key, uint32_t seen) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int r = lr + 4 * u;
      xk[u] = xv[u] = make_uint4(0, 0, 0, 0);
      if (seen >> r & 1) {
        xk[u] = *reinterpret_cast<const uint4*>(k + (int64_t)(key + r) * A.k.sn + cc * 8);
        xv[u] = *reinterpret_cast<const uint4*>(v + (int64_t)(key + r) * A.v.sn + cc * 8);
      }
    }
  };
  int key = range.x + wave * kBlock;
  uint32_t seen = seen_word(seen_byte(key));
  int next_byte = seen_byte(key + kBlock * kWaves);
  load(key, seen);
  for (; key < range.y; key += kBlock * kWaves) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      *reinterpret_cast<uint4*>(tk + (lr + 4 * u) * kStride + cc * 8) = xk[u];
      *reinterpret_cast<uint4*>(tv + (lr + 4 * u) * kStride + cc * 8) = xv[u];
    }
    // the wave's own LDS: its reads below follow its writes above, and those
    // the reads of the turn before (a wave's LDS operations stay in order; this
    // keeps the compiler from moving them past each other)
    asm volatile("" ::: "memory");
    const uint32_t now = seen;
    seen = seen_word(next_byte);
    load(key + kBlock * kWaves, seen);
    next_byte = seen_byte(key + 2 * kBlock * kWaves);
    f32x16 sc[1] = {scores(tk, qf, lane)};
    if (now != 0xffffffffu) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!(now >> (8 * (r >> 2) + 4 * hh + (r & 3)) & 1)) sc[0][r] = -__builtin_inff();
    }
    raise_max(x, sc, c);
    exponentials(x, sc[0], c);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const bf16x8 p = operand8(sc[0], y);
      x.l = add_bf16x8(p, x.l);
#pragma unroll
      for (int d = 0; d < 4; ++d) x.o[d] = mfma(column8(tv + 16 * y * kStride + 32 * d + tr), p, x.o[d]);
    }
    asm volatile("" ::: "memory");
  }

  // join the waves' rows
  __syncthreads();
  const float l = both_sum(x.l), exact = both_sum(x.exact);
  if (l32 < n_rows) {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(&lds.j.o[wave][l32][32 * d + 8 * q + 4 * hh]) =
            make_float4(x.o[d][4 * q], x.o[d][4 * q + 1], x.o[d][4 * q + 2], x.o[d][4 * q + 3]);
    if (hh == 0) {
      lds.j.m[wave][l32] = x.m;
      lds.j.l[wave][l32] = l;
      lds.j.exact[wave][l32] = exact;
    }
  }
  __syncthreads();
  const Parts p = parts_of(A.ws, (int64_t)s.B * s.H * s.N, nsplit);
  // one pair of dims of one row a thread and turn
  for (int i = t; i < n_rows * (D / 2); i += kFewThreads) {
    const int r = i / (D / 2), d = 2 * (i % (D / 2));
    const int hr = hk * per + (int)((row_base + r) / s.N), n = (int)((row_base + r) % s.N);
    if (n >= qlen) continue;
    float top = kNoMax, sum = 0.0f, exact_sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds.j.m[w][r]);
    float2 o = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f((lds.j.m[w][r] - top) * c);
      sum = __builtin_fmaf(f, lds.j.l[w][r], sum);
      exact_sum = __builtin_fmaf(f, lds.j.exact[w][r], exact_sum);
      o.x = __builtin_fmaf(f, lds.j.o[w][r][d], o.x);
      o.y = __builtin_fmaf(f, lds.j.o[w][r][d + 1], o.y);
    }
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    o.x *= inv;
    o.y *= inv;
    const int64_t at = ((int64_t)b * s.H + hr) * s.N + n;
    if (nsplit > 1) {
      const int64_t am = split * p.rows + at;
      *reinterpret_cast<float2*>(p.o + am * D + d) = o;
      if (d == 0) p.l[am] = log2_sum(top, sum, c);
      if (d == 0 && A.lse) p.exact[am] = log2_sum(top, exact_sum, c);
    } else {
      store_two(A, b, hr, n, d, o);
      if (A.lse && d == 0) A.lse[at] = log2_sum(top, exact_sum, c) * kLn2;
    }
  }
}

// The pieces' results joined: four waves take a row, two dims a lane.
__global__ __launch_bounds__(256) void cross_join_kernel(CrossFwd A, int pieces) {
  __shared__ float2 of[4][64];
  __shared__ float sums[4][3];
  lds_poison(of, sizeof(of));
  lds_poison(sums, sizeof(sums));
  lds_poison_done();
  const CrossShape& s = A.s;
  const int64_t rows = (int64_t)s.B * s.H * s.N, i = blockIdx.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int n = (int)(i % s.N), bh = (int)(i / s.N), h = bh % s.H, b = bh / s.H;
  if (n >= query_len(s, b)) return;
  const Parts p = parts_of(A.ws, rows, pieces);
  float top = kNoMax, sum = 0.0f, exact = 0.0f;
  // (loads of eight pieces at a time)
#pragma unroll 8
  for (int u = wave; u < pieces; u += 4) top = fmaxf(top, p.l[u * rows + i]);
  float2 o = make_float2(0.0f, 0.0f);
#pragma unroll 8
  for (int u = wave; u < pieces; u += 4) {
    const int64_t am = u * rows + i;
    const float f = __builtin_amdgcn_exp2f(p.l[am] - top);
    const float2 x = *reinterpret_cast<const float2*>(p.o + am * D + 2 * lane);
    sum += f;
    if (A.lse) exact += __builtin_amdgcn_exp2f(p.exact[am] - top);
    o.x = __builtin_fmaf(f, x.x, o.x);
    o.y = __builtin_fmaf(f, x.y, o.y);
  }
  of[wave][lane] = o;
  if (lane == 0) sums[wave][0] = top, sums[wave][1] = sum, sums[wave][2] = exact;
  __syncthreads();
  if (wave) return;
  top = fmaxf(fmaxf(sums[0][0], sums[1][0]), fmaxf(sums[2][0], sums[3][0]));
  sum = exact = 0.0f;
  o = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = __builtin_amdgcn_exp2f(sums[w][0] - top);
    sum = __builtin_fmaf(f, sums[w][1], sum);
    exact = __builtin_fmaf(f, sums[w][2], exact);
    o.x = __builtin_fmaf(f, of[w][lane].x, o.x);
    o.y = __builtin_fmaf(f, of[w][lane].y, o.y);
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  o.x *= inv;
  o.y *= inv;
  store_two(A, b, h, n, 2 * lane, o);
  if (A.lse && lane == 0) A.lse[i] = sum > 0.0f ? (top + log2f(exact)) * kLn2 : -__builtin_inff();
}

// ------------------------------------------------------ visible keys in order
//
// Where keys are masked the kernels that walk tiles of keys walk the visible ones alone:
// order[b] holds them first, in order, and then the others, counts[b] how many are visible.
// So a masked key costs no turn and is not read, and a sequence's visible keys are as a
// shorter sequence's, their rows found through order.  A workgroup goes through a sequence's
// mask, 1,024 keys a step of 1 us: 2.6 us for 333 keys, 11 for 12,480, 115 for 111,600.

constexpr int kOrderThreads = 1024;
__global__ __launch_bounds__(kOrderThreads) void cross_order_kernel(CrossShape s, int32_t* order, int32_t* counts) {
  __shared__ int waves[kOrderThreads / 64];
  const int b = blockIdx.x, t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int klen = key_len(s, b);
  const uint8_t* m = s.mask + (int64_t)b * s.M;
  int32_t* to = order + (int64_t)b * s.M;
  int seen = 0;  // visible keys before this step's
  for (int at = 0; at < s.M; at += kOrderThreads) {
    const int key = at + t;
    const bool on = key < klen && m[key] != 0;
    const uint64_t ones = __ballot(on);
    if (lane == 0) waves[wave] = __popcll(ones);
    __syncthreads();
    int before = seen, all = 0;
#pragma unroll
    for (int w = 0; w < kOrderThreads / 64; ++w) {
      if (w < wave) before += waves[w];
      all += waves[w];
    }
    before += __popcll(ones & ((1ull << lane) - 1));  // visible keys before this one
    if (key < s.M) to[on ? before : s.M - 1 - (key - before)] = key;  // (the others from the end)
    seen += all;
    __syncthreads();
  }
  if (t == 0) counts[b] = seen;
}

// A sequence's keys as the tile kernels walk them.
template <bool kMasked>
struct Keys {
  const int32_t* order;  // kMasked
  int len;
  Keys() = default;
  __device__ __forceinline__ Keys(const CrossShape& s, const int32_t* o, int b, int n) {
    order = kMasked ? o + (int64_t)b * s.M : nullptr;
    len = n;
  }
  __device__ __forceinline__ Keys(const CrossShape& s, const int32_t* o, const int32_t* counts, int b)
      : Keys(s, o, b, kMasked ? counts[b] : key_len(s, b)) {}
  __device__ __forceinline__ int at(int i) const { return kMasked ? order[i] : i; }
};

// Tiles of 32 keys and their values, one after the other from key `from` on, on their
// way into LDS, one kilobyte at a time: copy 0, 1 the halves of K's tile, 2, 3 V's.  A
// wave brings 8 rows.  Past the last tile it comes again, and is not used; keys past the
// sequence are its last one again (their scores are masked).  Masked keys' rows are
// looked up for eight tiles at a time, a lane each, and passed on by ds_bpermute: a
// look-up waits for all the copies before it (40 heads of 111,600 rows over 512 keys, all
// visible, looked up tile by tile 1,745 us, so 1,527; sooner, and waited for a tile later,
// 1,530).
constexpr int kTileKeys = 32;
constexpr int kRing = 4;
template <bool kMasked>
struct KeyCopies {
  const uint16_t *k, *v;  // the tile's first key (kMasked: the head's)
  int64_t ksn, vsn;
  Keys<kMasked> keys;
  int key, tile, turns, row, lane;
  uint32_t at, to_k, to_v, ok, ov;
  int rows, next;  // kMasked: rows of eight tiles, lane / 8 the tile; this lane's of the tile to come
  const uint16_t *mk, *mv;

  // n tiles from key `from` on.
  __device__ __forceinline__ void begin(const Rows& kr, const Rows& vr, int b, int hk, const Keys<kMasked>& ks, int from, int n,
                                        int wave, int l) {
    k = kr.p + b * kr.sb + hk * kr.sh;
    v = vr.p + b * vr.sb + hk * vr.sh;
    ksn = kr.sn;
    vsn = vr.sn;
    keys = ks;
    key = from;
    tile = 0;
    row = 8 * wave + (l >> 3);
    lane = l;
    turns = n;
    at = wave * kRowBlock;
    if (kMasked) {
      if (n > 0) look_up(0);
    } else {
      k += (int64_t)from * ksn;
      v += (int64_t)from * vsn;
      ok = copy_offset(row, ksn, lane);
      ov = copy_offset(row, vsn, lane);
    }
  }
  // kMasked: this lane's row of tile i, whose keys are from `key` on.
  __device__ __forceinline__ void look_up(int i) {
    if (i % 8 == 0) {
      rows = keys.order[min(key + kTileKeys * (lane >> 3) + (int)(at / kRowBlock) * 8 + (lane & 7), keys.len - 1)];
      asm volatile("" : "+v"(rows));  // (waited for here, not in every turn)
    }
    next = __builtin_amdgcn_ds_bpermute(4 * (i % 8 * 8 + (lane >> 3)), rows);
  }
  // The next tile (the first, to begin with) into LDS at k_to and v_to.
  __device__ __forceinline__ void start(uint32_t k_to, uint32_t v_to) {
    to_k = __builtin_amdgcn_readfirstlane(k_to + at);
    to_v = __builtin_amdgcn_readfirstlane(v_to + at);
    const bool on = tile > 0 && tile < turns;
    if (kMasked) {
      const int chunk = 8 * ((lane & 7) ^ swizzle(lane >> 3));
      mk = k + (int64_t)next * ksn + chunk;
      mv = v + (int64_t)next * vsn + chunk;
      if (tile + 1 < turns) {
        key += kTileKeys;
        look_up(tile + 1);
      }
    } else {
      key += on ? kTileKeys : 0;
      k += on ? kTileKeys * ksn : 0;
      v += on ? kTileKeys * vsn : 0;
      if (key + kTileKeys > keys.len) {
        const int r = min(row, keys.len - 1 - key);
        ok = copy_offset(r, ksn, lane);
        ov = copy_offset(r, vsn, lane);
      }
    }
    ++tile;
  }
  __device__ __forceinline__ void part(int n) const {
    const uint32_t lds = (n / 2 ? to_v : to_k) + n % 2 * 1024;
    if (kMasked) copy_1k_from(lds, (n / 2 ? mv : mk) + n % 2 * 64);
    else copy_1k(lds, n / 2 ? v : k, (n / 2 ? ov : ok) + n % 2 * 128);
  }
  __device__ __forceinline__ void all(uint32_t k_to, uint32_t v_to) {
    start(k_to, v_to);
#pragma unroll
    for (int n = 0; n < 4; ++n) part(n);
  }
};

// Tiles of 256 rows, a head's one after the other; where lengths differ head after
// head, so that every XCD has some of each sequence.
struct RowTile {
  int b, h, row0;
};
__host__ __device__ inline int tiles_of(int n, int rows) { return (n + rows - 1) / rows; }
__host__ __device__ inline int64_t row_tiles_of(const CrossShape& s) { return (int64_t)s.B * s.H * tiles_of(s.N, kCrossRows); }
__device__ __forceinline__ RowTile row_tile(int tile, const CrossShape& s) {
  const int per_head = tiles_of(s.N, kCrossRows), slab = tile / per_head;
  const int2 bh = slab_of(slab, s.H, s);
  return {bh.x, bh.y, (tile - slab * per_head) * kCrossRows};
}
// The tile and piece of a workgroup: tiles [0, full) whole, the rest in pieces; a run
// of consecutive ones to an XCD.
struct Piece {
  int tile, piece, pieces;
};
__device__ __forceinline__ Piece piece_of(int wg, int tiles, const DiffTiles& p) {
  if (wg < p.full) return {xcd_local_id(wg, p.full), 0, 1};
  const int id = xcd_local_id(wg - p.full, (tiles - p.full) * p.pieces);
  return {p.full + id / p.pieces, id % p.pieces, p.pieces};
}

// ----------------------------------------------------------- forward, row tiles

// The tile kernel's work is a line of turns: sequence after sequence, head after head,
// tile after tile of 256 rows, each as many turns as its keys make tiles of 32 (one
// where there is none).  Workgroup i of n takes turns [i total / n, (i + 1) total / n)
// of it, to the nearest tile's start unless tiles are split.  Lengths count where there
// are few sequences enough to add them up; else every sequence counts as a whole one.
constexpr int kMaxByLength = 1024;
// What a whole tile takes beside its keys' turns, while its rows come and go (3 x 16 heads
// of up to 4,097 rows over 333 masked keys 60 us where it counts for nothing, 49; 4 x 16 of
// 2,047 over 301 49, 38).  A split line has its turns alone.
constexpr int kTileTurns = 4;
struct Line {
  const CrossShape& s;
  const int32_t* counts;  // of visible keys, or null
  int tile_turns;         // turns that a tile counts for beside those of its keys; kEven: it is one
  bool by_length;
  static constexpr int kEven = -1;
  __device__ __forceinline__ Line(const CrossShape& sh, const int32_t* c, int per_tile) : s(sh), counts(c), tile_turns(per_tile) {
    by_length = (s.q_lens || s.kv_lens || s.mask) && s.B <= kMaxByLength;
  }
  __device__ __forceinline__ int keys(int b) const { return counts ? counts[b] : key_len(s, b); }
  __device__ __forceinline__ int tiles(int b) const { return tiles_of(by_length ? query_len(s, b) : s.N, kCrossRows); }
  __device__ __forceinline__ int turns(int b) const { return tile_turns == kEven ? 1 : tile_turns + max(1, tiles_of(by_length ? keys(b) : s.M, kTileKeys)); }
  __device__ __forceinline__ int64_t cost(int b) const { return (int64_t)s.H * tiles(b) * turns(b); }
};
struct Place {
  int b, h, rank, turn;
};
__device__ __forceinline__ Place place_in(const Line& l, int b, int64_t rest) {
  const int per_tile = l.turns(b);
  const int64_t tile = rest / per_tile, per_head = max(l.tiles(b), 1);
  return {b, (int)(tile / per_head), (int)(tile % per_head), (int)(rest - tile * per_tile)};
}
__device__ __forceinline__ Place uniform(const Place& p) {
  return {__builtin_amdgcn_readfirstlane(p.b), __builtin_amdgcn_readfirstlane(p.h), __builtin_amdgcn_readfirstlane(p.rank),
          __builtin_amdgcn_readfirstlane(p.turn)};
}
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)(((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32) | __builtin_amdgcn_readfirstlane((uint32_t)x));
}
__device__ __forceinline__ int64_t line_total(const Line& l) {
  if (!l.by_length) return l.cost(0) * l.s.B;
  const int lane = threadIdx.x & 63;
  int64_t total = 0;
  for (int b = lane; b < l.s.B; b += 64) total += l.cost(b);
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
  return uniform(total);
}
__device__ __forceinline__ Place find(const Line& l, int64_t turn, int64_t total) {
  const Place end = {l.s.B, 0, 0, 0};
  if (turn >= total) return end;
  if (!l.by_length) {
    const int64_t one = l.cost(0);
    return uniform(place_in(l, (int)(turn / one), turn % one));
  }
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int base = 0; base < l.s.B; base += 64) {
    const int b = base + lane;
    const int64_t mine = b < l.s.B ? l.cost(b) : 0;
    int64_t upto = mine;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int64_t x = __shfl_up(upto, m);
      if (lane >= m) upto += x;
    }
    const uint64_t past = __ballot(before + upto > turn);
    if (past) {
      const int at = __ffsll((unsigned long long)past) - 1;
      const int64_t start = before + uniform(__shfl(upto - mine, at));
      return uniform(place_in(l, base + at, turn - start));
    }
    before += uniform(__shfl(upto, 63));
  }
  return end;
}
// The next tile's start where the turn lies in a tile's second half, this one's otherwise.
__device__ __forceinline__ Place nearest(const Line& l, Place p) {
  if (p.b >= l.s.B || p.turn == 0) return p;
  if (2 * p.turn >= __builtin_amdgcn_readfirstlane(l.turns(p.b))) {
    if (++p.rank >= __builtin_amdgcn_readfirstlane(l.tiles(p.b))) {
      p.rank = 0;
      if (++p.h == l.s.H) {
        p.h = 0;
        do ++p.b;
        while (p.b < l.s.B && __builtin_amdgcn_readfirstlane(l.tiles(p.b)) == 0);  // (the next one's first tile is a place of the line)
      }
    }
  }
  p.turn = 0;
  return p;
}
// Workgroups that have a turn of the line.
__device__ __forceinline__ int line_workgroups(int64_t total, int launched) { return (int)min(total, (int64_t)launched); }
__device__ __forceinline__ int64_t line_bound(int64_t total, int i, int n) {
  return total / n * i + total % n * i / n;
}

// A workgroup's tiles one after the other: those with rows; turns `from` .. `to` of the
// current one are the workgroup's.
struct Tiles {
  Place at;
  int qlen, klen, from, to;
  int done;  // (as a bool the struct's copies went through scratch memory)
  __device__ __forceinline__ int turns() const { return tiles_of(klen, kTileKeys); }
  __device__ __forceinline__ bool whole() const { return from == 0 && to == turns(); }
  __device__ __forceinline__ int row0() const { return at.rank * kCrossRows; }
  __device__ __forceinline__ void lengths(const Line& l) {
    if (at.b >= l.s.B) return;
    qlen = __builtin_amdgcn_readfirstlane(query_len(l.s, at.b));
    klen = __builtin_amdgcn_readfirstlane(l.keys(at.b));
  }
  // From `at` on, the first tile that has rows and is not past `end` (which may name a
  // tile behind its sequence's rows, where lengths do not count).
  __device__ __forceinline__ void settle_on(const Line& l, const Place& end) {
    for (;;) {
      const bool end_head = at.b == end.b && at.h == end.h;
      if (at.b >= l.s.B || (end_head && (at.rank > end.rank || (at.rank == end.rank && at.turn >= end.turn)))) {
        done = true;
        return;
      }
      if (row0() < qlen) break;
      if (end_head) {
        done = true;
        return;
      }
      at.rank = at.turn = 0;
      if (++at.h == l.s.H) {
        at.h = 0;
        ++at.b;
        lengths(l);
      }
    }
    from = at.turn;
    to = turns();
    if (at.b == end.b && at.h == end.h && at.rank == end.rank) to = min(to, end.turn);
  }
  __device__ __forceinline__ void start(const Line& l, const Place& f, const Place& end) {
    at = f;
    done = false;
    qlen = klen = from = to = 0;
    lengths(l);
    settle_on(l, end);
  }
  __device__ __forceinline__ void next(const Line& l, const Place& end) {
    if (done) return;
    at.turn = 0;
    ++at.rank;
    settle_on(l, end);
  }
};

// Few keys (kShortKeys at most; a prompt's 77 tokens): all of a head's are in LDS, staged
// once for the tiles of it that a workgroup takes one after the other, so a tile is a read
// of its rows, a softmax and a write, and memory bounds it up to some 128 keys.  Eight
// waves of 32 rows, two a SIMD, that meet at a change of heads alone; a wave's next rows
// are on their way, in registers, while it works on the last.  Hidden keys are zeros in
// LDS, and not read.
//
// 40 heads of 111,600 rows: over 32 keys 468 us (4.9 TB/s of rows, as a copy), 77 476, 128
// 503, 192 586, 256 683 (860 TFLOP/s, as the tile kernel over more keys); the tile kernel,
// which has a tile's rows wait for memory no longer than its few turns, 663, 623, 587, 742,
// 852.  (Blocks of keys as a loop: 643 over 192, 760 over 256.)
constexpr int kShortWaves = kCrossRows / 32, kShortThreads = 64 * kShortWaves;
template <int kBlocks, bool kTrain>  // blocks of 32 keys
__global__ __launch_bounds__(kShortThreads) void cross_short_kernel(CrossFwd A) {
  struct Lds {
    uint8_t k[kBlocks][kTile32], v[kBlocks][kTile32];
    uint8_t out[kShortWaves][32 * D];  // half of the dims of a wave's rows, on their way out
  };
  __shared__ __attribute__((aligned(1024))) Lds lds;
  lds_poison(&lds, sizeof(lds));
  lds_poison_done();
  const CrossShape& s = A.s;
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  const int wg = xcd_local_id(blockIdx.x, gridDim.x), per = s.H / s.Hk;
  const float c = s.scale * kLog2e;
  const Line line(s, nullptr, Line::kEven);
  Place end;
  Tiles at, next;
  {
    const int64_t total = line_total(line);
    const int n = line_workgroups(total, gridDim.x);
    if (wg >= n) return;
    const Place from = find(line, line_bound(total, wg, n), total);
    end = find(line, line_bound(total, wg + 1, n), total);
    at.start(line, from, end);
  }
  bf16x8 q[8], q_next[8];
  auto load = [&](bf16x8(&f)[8], const Tiles& a) __attribute__((always_inline)) {
    const int n = a.row0() + 32 * wave + l32;
    load_row(f, A.q.p + a.at.b * A.q.sb + a.at.h * A.q.sh + (int64_t)n * A.q.sn, !a.done && n < a.qlen, hh);
  };
  uint32_t seen[kBlocks];  // visible keys, a bit each
  int held_b = -1, held_hk = -1;
  auto stage = [&](int b, int hk, int klen) __attribute__((always_inline)) {
    const uint16_t* k = A.k.p + b * A.k.sb + hk * A.k.sh;
    const uint16_t* v = A.v.p + b * A.v.sb + hk * A.v.sh;
    const int r = t >> 4, cc = t & 15;
    const int to = (r >> 3) * kRowBlock + (cc >> 3) * 1024 + (r & 7) * 128 + ((cc & 7) ^ swizzle(r)) * 16;
    constexpr int kStep = kBlocks < 4 ? kBlocks : 4;
#pragma unroll
    for (int from = 0; from < kBlocks; from += kStep) {
      uint4 xk[kStep], xv[kStep];
#pragma unroll
      for (int w = 0; w < kStep; ++w) {
        const int u = from + w, key = 32 * u + l32;
        seen[u] = (uint32_t)__ballot(key < klen && (!s.mask || s.mask[(int64_t)b * s.M + key] != 0));
        xk[w] = xv[w] = make_uint4(0, 0, 0, 0);
        if (seen[u] >> r & 1) {
          xk[w] = *reinterpret_cast<const uint4*>(k + (int64_t)(32 * u + r) * A.k.sn + 8 * cc);
          xv[w] = *reinterpret_cast<const uint4*>(v + (int64_t)(32 * u + r) * A.v.sn + 8 * cc);
        }
      }
      if (from == 0) __syncthreads();  // the last head's are done with
#pragma unroll
      for (int w = 0; w < kStep; ++w) {
        *reinterpret_cast<uint4*>(lds.k[from + w] + to) = xk[w];
        *reinterpret_cast<uint4*>(lds.v[from + w] + to) = xv[w];
      }
    }
    __syncthreads();
  };
  // The wave's rows to memory, 64 dims at a time through its LDS: the 16-byte chunk c of
  // row r lies at place c ^ (r % 8), so that 8 lanes write 128 bytes of a row.
  auto store_halves = [&](uint16_t* to, int64_t sn, int rows, auto&& words) __attribute__((always_inline)) {
    uint8_t* mine = lds.out[wave];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int z = 0; z < 4; ++z)
          *reinterpret_cast<uint2*>(mine + l32 * D + 16 * ((4 * d + z) ^ (l32 & 7)) + 8 * hh) = words(2 * half + d, z);
      asm volatile("" ::: "memory");  // the wave's LDS operations stay in order
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int r = 8 * u + (lane >> 3), cc = lane & 7;
        const uint4 x = *reinterpret_cast<const uint4*>(mine + r * D + 16 * (cc ^ (r & 7)));
        if (r < rows) *reinterpret_cast<uint4*>(to + (int64_t)r * sn + 64 * half + 8 * cc) = x;
      }
      asm volatile("" ::: "memory");
    }
  };
  const RowPlace rp = row_place(lane);
  const int cp = col_place(lane);
  load(q_next, at);
  while (!at.done) {
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) q[kk] = q_next[kk];
    next = at;
    next.next(line, end);
    const int b = at.at.b, h = at.at.h, hk = h / per, first = at.row0() + 32 * wave;
    if (b != held_b || hk != held_hk) {
      held_b = b;
      held_hk = hk;
      stage(b, hk, at.klen);
    }
    load(q_next, next);
    if (first < at.qlen) {
      MapRows x;
      clear(x);
#pragma unroll
      for (int u = 0; u < kBlocks; ++u) {
        if (u > 0 && 32 * u >= at.klen) break;
        f32x16 sc[1] = {};
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) sc[0] = mfma(row_frag(lds.k[u], rp, kk), q[kk], sc[0]);
        if (seen[u] != 0xffffffffu) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (!(seen[u] >> (8 * (r >> 2) + 4 * hh + (r & 3)) & 1)) sc[0][r] = -__builtin_inff();
        }
        raise_max(x, sc, c);
        exponentials(x, sc[0], c);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const bf16x8 p = operand8(sc[0], y);
          x.l = add_bf16x8(p, x.l);
#pragma unroll
          for (int d = 0; d < 4; ++d) x.o[d] = mfma(col_frag(lds.v[u] + cp, y, d), p, x.o[d]);
        }
      }
      const float l = both_sum(x.l), inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) x.o[d][r] *= inv;
      const int rows = at.qlen - first;
      if (kTrain) {
        const int64_t row = ((int64_t)b * s.H + h) * s.N + first;
        const float lse = log2_sum(x.m, both_sum(x.exact), c) * kLn2;
        if (hh == 0 && l32 < rows) A.lse[row + l32] = lse;
        store_halves(A.left + row * D, D, rows, [&](int d, int z) { return left4(x.o[d], z, pack4(x.o[d], z)); });
      }
      store_halves(A.out.p + b * A.out.sb + h * A.out.sh + (int64_t)first * A.out.sn, A.out.sn, rows,
                   [&](int d, int z) { return pack4(x.o[d], z); });
    }
    at = next;
  }
}

// Where workgroup `wg` of a split line leaves its share of a tile: before one that
// another began (0), or after the last that it began itself (1); 256 rows of 128 and
// two logarithms each.
constexpr int kShareFloats = kCrossRows * (D + 2);
__device__ __forceinline__ float* share_of(float* ws, int wg, bool began) {
  return ws + ((int64_t)2 * wg + began) * kShareFloats;
}

// 256 rows of one head a tile, 64 a wave in two blocks of 32 (a fragment of K or V is
// read once for two MFMAs); one wave a SIMD, so its MFMAs, exponentials and LDS reads
// have to overlap inside the wave: a turn of the loop is a list of slots, each an MFMA,
// the LDS read of a fragment some slots on and a share of the arithmetic on scores that
// are done, and nothing moves between slots.  Turn i: the products P V of item i - 1,
// the exponentials of item i, the scores of item i + 1, an item being 32 keys of a tile.
// Items follow each other over the tiles' borders, so that a tile of few keys (a
// prompt's 512 are 16 turns) pays for no pipeline of its own: its rows come into LDS
// while the tile before is walked, and its outputs leave while the next one's copies
// are on their way.
//
// A row is held to the maximum of its first item: P and the sums have 8 exponent bits,
// so scores far above it cost no precision, and most rows' stay within a few binades.
// A row whose P add up to more than 2^80 (55 above it in the exponent), or whose
// products with the values leave fp32, has its wave walk the tile again by itself,
// raising the maxima as they come.
constexpr float kTooMuch = 1.2089258e24f;
template <bool kMasked, bool kTrain>
__global__ __launch_bounds__(256, 1) void cross_fwd_kernel(CrossFwd A, bool split) {
  constexpr int kFrags = 16, kAhead = 6, kHold = 8;
  // A turn reads V of item i - 1 and K of item i + 1 and sends for item i + kLook, in four
  // copies; items of a tile: an even number, kLook at least (past its keys the last one
  // again, masked), so that copies reach no further than into the next tile.
  constexpr int kLook = 4, kKPlaces = 4, kVPlaces = 8;
  struct Lds {
    uint8_t k[kKPlaces][kTile32], v[kVPlaces][kTile32];
    uint8_t rows[4][2][kTile32];  // of each wave: the next tile's q, or an output on its way
  };
  __shared__ __attribute__((aligned(1024))) Lds lds;
  lds_poison(&lds, sizeof(lds));
  lds_poison_done();
  const CrossShape& s = A.s;
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  const int wg = xcd_local_id(blockIdx.x, gridDim.x), per = s.H / s.Hk;
  const float c = s.scale * kLog2e;
  const Line line(s, kMasked ? A.counts : nullptr, split ? 0 : kTileTurns);
  Place end;
  Tiles now_at, next_at;
  {
    const int64_t total = line_total(line);
    const int n = line_workgroups(total, gridDim.x);
    if (wg >= n) return;
    Place from = find(line, line_bound(total, wg, n), total);
    end = find(line, line_bound(total, wg + 1, n), total);
    if (!split) {
      from = nearest(line, from);
      end = nearest(line, end);
    }
    now_at.start(line, from, end);
  }

  // This lane, where what follows from it is to be found there and not kept (in registers
  // that the turns need) from the kernel's start on.
  auto lane_here = []() __attribute__((always_inline)) {
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(l));
    return l;
  };
  // outputs of rows without keys: their tile has no turns
  auto no_keys = [&](const Tiles& at) __attribute__((always_inline)) {
    uint16_t* to = A.out.p + at.at.b * A.out.sb + at.at.h * A.out.sh;
    const int64_t row = ((int64_t)at.at.b * s.H + at.at.h) * s.N;
    const int t = 64 * wave + lane_here();
    for (int i = t; i < kCrossRows * kChunks; i += 256) {
      const int n = at.row0() + i / kChunks, cc = i % kChunks;
      if (n >= at.qlen) break;
      *reinterpret_cast<uint4*>(to + (int64_t)n * A.out.sn + 8 * cc) = make_uint4(0, 0, 0, 0);
      if (kTrain) *reinterpret_cast<uint4*>(A.left + (row + n) * D + 8 * cc) = make_uint4(0, 0, 0, 0);
      if (kTrain && cc == 0) A.lse[row + n] = -__builtin_inff();
    }
  };
  // on to a tile that has turns; those without are written on the way
  auto to_turns = [&](Tiles& at) __attribute__((always_inline)) {
    while (!at.done && at.from >= at.to) {
      if (at.klen == 0) no_keys(at);
      at.next(line, end);
    }
  };
  to_turns(now_at);
  if (now_at.done) return;

  // the items' copies: now_at's, then the next tile's
  KeyCopies<kMasked> copy;
  auto copy_tile = [&](const Tiles& at) __attribute__((always_inline)) {
    copy.begin(A.k, A.v, at.at.b, at.at.h / per, Keys<kMasked>(s, A.order, at.at.b, at.klen), at.from * kTileKeys,
               at.to - at.from, wave, lane);
  };
  int item = 0;  // of all, at the tile's start
  auto k_place = [&](int i) __attribute__((always_inline)) { return &lds.k[(item + i) % kKPlaces][0]; };
  auto v_place = [&](int i) __attribute__((always_inline)) { return &lds.v[(item + i) % kVPlaces][0]; };

  // The wave's 64 rows in LDS, 16 KB, at a tile's end: first its outputs on their way to
  // memory, then the q of the tile after the next on its way from there.  Both are
  // exactly 16 operations of the wave (outputs of training twice 16 and two log sums):
  // rows behind the sequence are its last one again, of q and so of the outputs, which the
  // wave that has that row stores over it, the same bits.  So a turn knows what was sent for
  // after the copies that it needs, and waits for nothing else: memory has three turns for
  // the rows.  (A wave whose rows all lie behind the sequence stores none of them: the last
  // row's own wave may walk again, and round otherwise.)
  constexpr int kRowOps = kTrain ? 50 : 32;
  uint8_t* mine = &lds.rows[wave][0][0];
  auto mine_at = [&]() __attribute__((always_inline)) { return lds_address(&lds.rows[0][0][0]) + wave * (uint32_t)sizeof(lds.rows[0]); };
  // Row r's 16-byte chunk c of an output lies at place c ^ (r % 16), its halves exchanged
  // for odd r / 16: written 8 bytes a lane, a row a lane, and read a row a 16 lanes, without
  // bank conflicts.
  auto stage = [&](int m, auto&& words) __attribute__((always_inline)) {
    const int lane = lane_here(), hh = lane >> 5, l32 = lane & 31;
    uint8_t* row = mine + (32 * m + l32) * 2 * D + 8 * (hh ^ (l32 >> 4));
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q) *reinterpret_cast<uint2*>(row + 16 * ((4 * d + q) ^ (l32 & 15))) = words(d, q);
  };
  auto store_staged = [&](uint16_t* to, int64_t sn, int last) __attribute__((always_inline)) {
    const int lane = lane_here();
    asm volatile("" ::: "memory");  // the wave's LDS operations stay in order
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      const int r = 4 * u + (lane >> 4);
      const uint4 y = *reinterpret_cast<const uint4*>(mine + r * 2 * D + 16 * ((lane & 15) ^ (r & 15)));
      *reinterpret_cast<uint4*>(to + (int64_t)min(64 * wave + r, last) * sn + 8 * (lane & 15)) =
          4 * u & 16 ? make_uint4(y.z, y.w, y.x, y.y) : y;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  auto copy_rows = [&](const Tiles& at) __attribute__((always_inline)) {
    const int lane = lane_here();
    const uint16_t* q = A.q.p + at.at.b * A.q.sb + at.at.h * A.q.sh + (int64_t)at.row0() * A.q.sn + 8 * ((lane & 7) ^ swizzle(lane >> 3));
    const int last = at.qlen - 1 - at.row0();
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const uint16_t* p = q + (int64_t)min(64 * wave + 8 * u + (lane >> 3), last) * A.q.sn;
      const uint32_t to = __builtin_amdgcn_readfirstlane(mine_at() + u * kRowBlock);
      copy_1k_from(to, p);
      copy_1k_from(to + 1024, p + 64);
    }
  };
  bf16x8 qf[2][8];
  const RowPlace rp = row_place(lane);
  const int cp = col_place(lane);
  auto load_rows = [&]() __attribute__((always_inline)) {
    // the wave's own copies: three turns' at least were sent for after them
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * (kLook - 1)) : "memory");
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) qf[m][kk] = row_frag(mine + m * kTile32, rp, kk);
    asm volatile("" ::: "memory");
    hold_in_agprs(qf[0]);
    hold_in_agprs(qf[1]);
  };

  struct Item {
    f32x16 s[2];        // scores of the row blocks
    uint32_t pw[2][8];  // P, packed
  } ia, ib;
  MapRows x[2];
  float mc[2];  // the maxima held to, times c
  bf16x8 ring[kHold];
  int n_turns = 0, n_items = 0, n_keys = 0, key0 = 0;  // items with keys, and all of the tile
  // the fragments of a turn in order: V of item i - 1, then K of item i + 1
  auto fragment = [&](int f, const uint8_t* v, const uint8_t* k) __attribute__((always_inline)) {
    return f < 8 ? col_frag(v + cp, f >> 2, f & 3) : row_frag(k, rp, f - 8);
  };
  auto mask_item = [&](Item& now, int i) __attribute__((always_inline)) {
    const int key = key0 + i * kTileKeys;
    if (key + kTileKeys > n_keys || i >= n_turns) {
      const int last = i < n_turns ? n_keys - 1 : -1;
      settle(now.s[0], now.s[1]);
      mask(now.s[0], key + 4 * hh, last);
      mask(now.s[1], key + 4 * hh, last);
    }
  };
  // one exponential; its pair is summed and packed with the next one's (an
  // exponential's result is not there at once)
  float e[2];
  auto take = [&](Item& now, int m, int r) __attribute__((always_inline)) {  // keys r, r + 1
    if (kTrain) x[m].exact += e[0];
    now.pw[m][r >> 1] = pack_bf16x2(e[0], e[1]);
    if (kTrain) x[m].exact += e[1];
    pin(now.pw[m][r >> 1]);
    x[m].l = add_bf16x2(now.pw[m][r >> 1], x[m].l);
    pin(x[m].l);
    if (kTrain) pin(x[m].exact);
  };
  auto exponential = [&](Item& now, int m, int r) __attribute__((always_inline)) {
    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(now.s[m][r], c, -mc[m]));
    if (r % 2 == 0 && r > 0) take(now, m, r - 2);
    if (r == 0 && m == 1) take(now, 0, 14);
    e[r & 1] = p;
    pin(e[r & 1]);
  };
  auto operand = [&](const Item& z, int m, int y) __attribute__((always_inline)) {
    return __builtin_bit_cast(bf16x8, make_uint4(z.pw[m][4 * y], z.pw[m][4 * y + 1], z.pw[m][4 * y + 2], z.pw[m][4 * y + 3]));
  };
  // Item i of the tile; old: item i - 1's P, and room for the next item's scores (after the
  // last one the next tile's first).
  auto turn = [&](int i, Item& now, Item& old) __attribute__((always_inline)) {
    const uint8_t* then = v_place(max(i - 1, 0));  // (turn 0's products are of P = 0)
    const uint8_t* here = v_place(i);
    const uint8_t* next = k_place(i + 1);
    mask_item(now, i);
#pragma unroll
    for (int d = 0; d < 4; ++d) asm volatile("" : "+a"(x[0].o[d]), "+a"(x[1].o[d]));
    hold_in_agprs(qf[0]);
    hold_in_agprs(qf[1]);
    each<0, 32>([&](auto slot) __attribute__((always_inline)) {
      constexpr int j = slot.value, f = j / 2, m = j & 1;
      if constexpr (j == 2) {
        // the next item, sent for three turns ago: after it two turns' copies, and in a
        // tile's first three turns the rows'
        if (i < kLook - 1) copies_landed<4 * (kLook - 2) + kRowOps>();
        else copies_landed<4 * (kLook - 2)>();
        if (i + kLook == n_items && !next_at.done) copy_tile(next_at);  // (past the last tile its last item again)
        copy.start(lds_address(k_place(i + kLook)), lds_address(v_place(i + kLook)));
        slot_end();
      }
      if constexpr (j >= 3 && j < 7) copy.part(j - 3);
      if constexpr (j < 16) {
        constexpr int d = f & 3, y = j >> 3;
        x[m].o[d] = mfma(ring[f % kHold], operand(old, m, y), x[m].o[d]);
      } else {
        constexpr int kk = f - 8;
        if constexpr (kk == 0) score_first_a(old.s[m], ring[f % kHold], qf[m][kk]);
        else score_a(old.s[m], ring[f % kHold], qf[m][kk]);
      }
      if constexpr (m == 0) {
        constexpr int g = f + kAhead;
        ring[g % kHold] = g < kFrags ? fragment(g, then, next) : fragment(g - kFrags, here, nullptr);
      }
      if constexpr (j >= 2 && j < 16) {
#pragma unroll
        for (int u = (j - 2) * 8 / 7; u < (j - 1) * 8 / 7; ++u) exponential(now, 0, u);
      }
      if constexpr (j >= 16) exponential(now, 1, j - 16);
      slot_end();
    });
    take(now, 1, 14);
  };
  auto last_products = [&](const Item& old) __attribute__((always_inline)) {
    const uint8_t* then = v_place(n_items - 1);
#pragma unroll
    for (int f = 0; f < 8; ++f) {
      const bf16x8 v = f < kAhead ? ring[f % kHold] : fragment(f, then, nullptr);
#pragma unroll
      for (int m = 0; m < 2; ++m) x[m].o[f & 3] = mfma(v, operand(old, m, f >> 2), x[m].o[f & 3]);
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
    return __any(top >= 0x7f800000u) != 0;
  };
  // o of 32 rows divided by their sums; of those, for the workspace or for training, the
  // log2 of the sums
  auto divide = [&](MapRows& y) __attribute__((always_inline)) {
    const float inv = 1.0f / both_sum(y.l);  // (a row behind the sequence is its last one again)
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) y.o[d][r] *= inv;
  };
  // a share of a tile, 32 rows from its row `first` on, to the workspace
  auto store_share = [&](const Tiles& at, int first, const MapRows& y, float held) __attribute__((always_inline)) {
    const int lane = lane_here(), hh = lane >> 5, l32 = lane & 31;
    float* share = share_of(A.ws, wg, at.from == 0);
    float* to = share + (first + l32) * D + 4 * hh;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(to + 32 * d + 8 * q) =
            make_float4(y.o[d][4 * q], y.o[d][4 * q + 1], y.o[d][4 * q + 2], y.o[d][4 * q + 3]);
    const float l2 = held + log2f(both_sum(y.l)), exact2 = kTrain ? held + log2f(both_sum(y.exact)) : 0.0f;
    if (hh == 0) share[kCrossRows * D + first + l32] = l2;
    if (kTrain && hh == 0) share[kCrossRows * (D + 1) + first + l32] = exact2;
  };
  // A tile's outputs.  (All is there when the turns that count the rows' operations come:
  // those of a share are not counted, and waited for.)
  auto finish = [&](const Tiles& at) __attribute__((always_inline)) {
    divide(x[0]);
    divide(x[1]);
    if (!at.whole()) {
      store_share(at, 64 * wave, x[0], mc[0]);
      store_share(at, 64 * wave + 32, x[1], mc[1]);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      return;
    }
    const int last = at.qlen - 1 - at.row0();
    if (kTrain) {
      const int64_t row = ((int64_t)at.at.b * s.H + at.at.h) * s.N + at.row0();
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const float lse = (mc[m] + log2f(both_sum(x[m].exact))) * kLn2;
        if (hh == 0) A.lse[row + min(64 * wave + 32 * m + l32, last)] = lse;
        stage(m, [&](int d, int q) { return left4(x[m].o[d], q, pack4(x[m].o[d], q)); });
      }
      store_staged(A.left + row * D, D, last);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) stage(m, [&](int d, int q) { return pack4(x[m].o[d], q); });
    store_staged(A.out.p + at.at.b * A.out.sb + at.at.h * A.out.sh + (int64_t)at.row0() * A.out.sn, A.out.sn, last);
  };
  // The wave's rows of a tile again, the running maxima raised as they come: the wave by
  // itself, its rows' place for the tiles of keys, and the outputs straight to memory.
  auto again = [&](const Tiles& at) __attribute__((always_inline)) {
    const int lane = lane_here(), hh = lane >> 5, l32 = lane & 31;
    const RowPlace rp = row_place(lane);
    const int cp = col_place(lane);
    const Keys<kMasked> keys(s, A.order, at.at.b, at.klen);
    const int chunk = 8 * ((lane & 7) ^ swizzle(lane >> 3));
    const uint16_t* k = A.k.p + at.at.b * A.k.sb + at.at.h / per * A.k.sh + chunk;
    const uint16_t* v = A.v.p + at.at.b * A.v.sb + at.at.h / per * A.v.sh + chunk;
#pragma unroll 1
    for (int first = 64 * wave; first < 64 * wave + 64; first += 32) {
      bf16x8 rows[8];
      MapRows y;
      clear(y);
      load_row(rows, A.q.p + at.at.b * A.q.sb + at.at.h * A.q.sh + (int64_t)min(at.row0() + first + l32, at.qlen - 1) * A.q.sn,
               true, hh);
#pragma unroll 1
      for (int key = at.from * kTileKeys; key < min(at.to * kTileKeys, at.klen); key += kTileKeys) {
#pragma unroll 1
        for (int u = 0; u < 4; ++u) {
          const int64_t r = keys.at(min(key + 8 * u + (lane >> 3), at.klen - 1));
          const uint32_t to = __builtin_amdgcn_readfirstlane(mine_at() + u * kRowBlock);
          copy_1k_from(to, k + r * A.k.sn);
          copy_1k_from(to + 1024, k + r * A.k.sn + 64);
          copy_1k_from(to + kTile32, v + r * A.v.sn);
          copy_1k_from(to + kTile32 + 1024, v + r * A.v.sn + 64);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        f32x16 sc[1] = {};
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) sc[0] = mfma(row_frag(mine, rp, kk), rows[kk], sc[0]);
        mask(sc[0], key + 4 * hh, at.klen - 1);
        raise_max(y, sc, c);
        exponentials(y, sc[0], c);
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const bf16x8 p = operand8(sc[0], z);
          y.l = add_bf16x8(p, y.l);
#pragma unroll
          for (int d = 0; d < 4; ++d) y.o[d] = mfma(col_frag(mine + kTile32 + cp, z, d), p, y.o[d]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the place's reads, before the next copies
      }
      divide(y);
      if (!at.whole()) {
        store_share(at, first, y, y.m * c);
        continue;
      }
      const int n = at.row0() + first, rows_left = at.qlen - n;
      const int64_t row = ((int64_t)at.at.b * s.H + at.at.h) * s.N + n;
      if (kTrain) {
        const float lse = (y.m * c + log2f(both_sum(y.exact))) * kLn2;
        if (hh == 0 && l32 < rows_left) A.lse[row + l32] = lse;
        store_rows(mine, lane, A.left + row * D, D, 0, rows_left, [&](int d, int q) { return left4(y.o[d], q, pack4(y.o[d], q)); });
      }
      store_rows(mine, lane, A.out.p + at.at.b * A.out.sb + at.at.h * A.out.sh + (int64_t)n * A.out.sn, A.out.sn, 0, rows_left,
                 [&](int d, int q) { return pack4(y.o[d], q); });
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // (not counted)
  };

  copy_rows(now_at);
  copy_tile(now_at);
#pragma unroll
  for (int u = 0; u < kLook; ++u) copy.all(lds_address(k_place(u)), lds_address(v_place(u)));
  next_at = now_at;
  next_at.next(line, end);
  to_turns(next_at);
  copies_landed<0>();
  load_rows();
  all_landed();
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) {
    const bf16x8 f = row_frag(k_place(0), rp, kk);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      if (kk == 0) score_first_a(ia.s[m], f, qf[m][kk]);
      else score_a(ia.s[m], f, qf[m][kk]);
    }
  }
  for (;;) {
    copy_rows(next_at.done ? now_at : next_at);  // (of no use where there is none, but of the same number)
    n_turns = now_at.to - now_at.from;
    n_items = max(n_turns + (n_turns & 1), kLook);
    n_keys = now_at.klen;
    key0 = now_at.from * kTileKeys;
    settle(ia.s[0], ia.s[1]);
    mask_item(ia, 0);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float top = ia.s[m][0];
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(top, ia.s[m][r]);
      clear(x[m]);
      mc[m] = both_max(top) * c;
#pragma unroll
      for (int w = 0; w < 8; ++w) ib.pw[m][w] = 0;
    }
#pragma unroll
    for (int f = 0; f < kAhead; ++f) ring[f] = fragment(f, v_place(0), nullptr);
    for (int i = 0; i < n_items; i += 2) {
      turn(i, ia, ib);
      if (i + 2 == n_items) load_rows();  // the next tile's, whose first scores the last turn finds
      turn(i + 1, ib, ia);
    }
    last_products(ib);
    if (now_at.row0() + 64 * wave >= now_at.qlen) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no row of its own (not counted)
    else if (__any(!(x[0].l < kTooMuch && x[1].l < kTooMuch)) != 0 || not_finite()) again(now_at);
    else finish(now_at);
    item += n_items;
    now_at = next_at;
    if (now_at.done) break;
    next_at.next(line, end);
    to_turns(next_at);
  }
  copies_landed<0>();  // none is under way when the wave ends
}

// Tiles that workgroups shared, joined: 16 rows of a tile a workgroup, a row's 16
// chunks of 8 dims a lane each.
__global__ __launch_bounds__(256) void cross_shares_kernel(CrossFwd A, int launched) {
  const CrossShape& s = A.s;
  const Line line(s, s.mask ? A.counts : nullptr, 0);
  const int per_head = tiles_of(s.N, kCrossRows), steps = kCrossRows / 16;
  const int tile = blockIdx.x / steps, r = blockIdx.x % steps * 16 + (threadIdx.x >> 4), cc = threadIdx.x & 15;
  const int rank = tile % per_head, bh = tile / per_head, h = bh % s.H, b = bh / s.H;
  const int n = rank * kCrossRows + r, qlen = query_len(s, b);
  if (rank * kCrossRows >= qlen) return;
  // the tile's turns in the line, and the first and last workgroup that has some
  const int64_t total = line_total(line), turns = line.turns(b);
  const int wgs = line_workgroups(total, launched);
  int64_t at = ((int64_t)h * line.tiles(b) + rank) * turns;
  if (line.by_length) {
    int64_t before = 0;
    for (int i = threadIdx.x & 63; i < b; i += 64) before += line.cost(i);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) before += __shfl_xor(before, m);
    at += before;
  } else {
    at += b * line.cost(0);
  }
  const int w0 = (int)(((at + 1) * wgs - 1) / total), w1 = (int)(((at + turns) * wgs - 1) / total);
  if (w0 == w1 || n >= qlen) return;
  auto share = [&](int w) { return share_of(A.ws, w, w == w0); };  // (the first has the tile's first turn, no other one)
  float top = kNoMax;
  for (int w = w0; w <= w1; ++w) top = fmaxf(top, share(w)[kCrossRows * D + r]);
  float sum = 0.0f, exact = 0.0f, o[8] = {};
  for (int w = w0; w <= w1; ++w) {
    const float* x = share(w);
    const float f = __builtin_amdgcn_exp2f(x[kCrossRows * D + r] - top);
    sum += f;
    if (A.lse) exact += __builtin_amdgcn_exp2f(x[kCrossRows * (D + 1) + r] - top);
    const float4 a = *reinterpret_cast<const float4*>(x + r * D + 8 * cc), z = *reinterpret_cast<const float4*>(x + r * D + 8 * cc + 4);
    o[0] = __builtin_fmaf(f, a.x, o[0]); o[1] = __builtin_fmaf(f, a.y, o[1]);
    o[2] = __builtin_fmaf(f, a.z, o[2]); o[3] = __builtin_fmaf(f, a.w, o[3]);
    o[4] = __builtin_fmaf(f, z.x, o[4]); o[5] = __builtin_fmaf(f, z.y, o[5]);
    o[6] = __builtin_fmaf(f, z.z, o[6]); o[7] = __builtin_fmaf(f, z.w, o[7]);
  }
  const float inv = 1.0f / sum;
#pragma unroll
  for (int u = 0; u < 8; ++u) o[u] *= inv;
  const uint4 y = pack_bf16x8(o);
  *reinterpret_cast<uint4*>(A.out.p + b * A.out.sb + h * A.out.sh + (int64_t)n * A.out.sn + 8 * cc) = y;
  if (A.lse) {
    const int64_t row = (int64_t)bh * s.N + n;
    *reinterpret_cast<uint4*>(A.left + row * D + 8 * cc) =
        make_uint4(left2(o[0], o[1], y.x), left2(o[2], o[3], y.y), left2(o[4], o[5], y.z), left2(o[6], o[7], y.w));
    if (cc == 0) A.lse[row] = (top + log2f(exact)) * kLn2;
  }
}

// ------------------------------------------------------------------ backward
//
// With X = dout v^T, P the probabilities and delta = dout . out of a row,
//   dS = P (X - delta),  dq = scale dS k,  dk = scale dS^T q,  dv = P^T dout.
// P is found again from the rows' log sums.  dS and P are rounded to bf16 for their
// products with k, q and dout, which are bf16: a result's error is its terms'
// roundings and its own, of one size (0.0024 of its norm together).  Two halves, one
// that owns rows (dq) and one that owns keys (dk, dv): no atomics, and every sum in
// a fixed order.

// What the backward kernels know of a row, 32 rows together: kStatLse: -lse / scale,
// which added to raw scores and scaled gives log2 P (-inf, and so P = 0, where the
// row has no keys or is not the sequence's); kStatDelta: -delta; 32 floats each.
constexpr int kBwdRows = 32;
constexpr int kStatFloats = 2 * kBwdRows;
enum { kStatLse = 0, kStatDelta = kBwdRows };

__global__ __launch_bounds__(16 * kBwdRows) void cross_stats_kernel(CrossBwd A) {
  const CrossShape& s = A.s;
  const int row_tiles = tiles_of(s.N, kBwdRows);
  const int r = threadIdx.x >> 4, cc = threadIdx.x & 15;
  const int n = (int)(blockIdx.x % row_tiles) * kBwdRows + r;
  const int bh = blockIdx.x / row_tiles, h = bh % s.H, b = bh / s.H;
  const bool valid = n < query_len(s, b);
  float d = 0.0f;
  if (valid) {
    float o[8], g[8], left[8];
    auto load = [](float (&f)[8], const uint16_t* p) { unpack_bf16x8(*reinterpret_cast<const uint4*>(p), f); };
    load(o, A.out.p + b * A.out.sb + h * A.out.sh + (int64_t)n * A.out.sn + 8 * cc);
    load(g, A.dout.p + b * A.dout.sb + h * A.dout.sh + (int64_t)n * A.dout.sn + 8 * cc);
    load(left, A.left + ((int64_t)bh * s.N + n) * D + 8 * cc);
#pragma unroll
    for (int u = 0; u < 8; ++u) d = __builtin_fmaf(g[u], o[u] + left[u], d);
  }
  d = row_sumsq_lanes16(d);
  if (cc < 2) {
    const float lse = valid ? A.lse[(int64_t)bh * s.N + n] : 0.0f;
    const bool some = valid && lse > -3e38f;
    A.stats[(int64_t)blockIdx.x * kStatFloats + cc * kBwdRows + r] =
        cc ? (some ? -d : 0.0f) : some ? -lse / s.scale : -__builtin_inff();
  }
}

// A backward turn t finds the scores and X of tile t, the exponentials of tile t
// (from the slot where its scores are done), what is left of tile t - 1 to its
// operands, and the gradient products of tile t - 1.  The barrier stands where the
// last eight slots begin, so that the next tile's first fragments are read before
// the turn ends.

// dq of 256 rows of one head, 64 a wave in two blocks of 32 (a fragment of K or V is
// read once for two MFMAs), over all the keys.
template <bool kMasked>
__device__ __forceinline__ void dq_of(const CrossBwd& A, uint8_t (*lds)[2][kTile32], int wg) {
  constexpr int kAhead = 6, kHold = 8;
  const CrossShape& s = A.s;
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  const Piece pc = piece_of(wg, (int)row_tiles_of(s), A.plan);
  const RowTile rt = row_tile(pc.tile, s);
  const int b = rt.b, h = rt.h, hk = h / (s.H / s.Hk);
  const int qlen = query_len(s, b);
  const Keys<kMasked> keys(s, A.order, A.counts, b);
  const int row = rt.row0 + 64 * wave + l32;  // and 32 more
  const float c = s.scale * kLog2e;

  bf16x8 qf[2][8], gf[2][8];
  float lse[2], del[2];
  const int row_tiles = tiles_of(s.N, kBwdRows);
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const int n = row + 32 * m;
    const bool valid = n < qlen;
    load_row(qf[m], A.q.p + b * A.q.sb + h * A.q.sh + (int64_t)n * A.q.sn, valid, hh);
    load_row(gf[m], A.dout.p + b * A.dout.sb + h * A.dout.sh + (int64_t)n * A.dout.sn, valid, hh);
    lse[m] = -__builtin_inff();
    del[m] = 0.0f;
    if (valid) {
      const float* st = A.stats + ((int64_t)(b * s.H + h) * row_tiles + n / kBwdRows) * kStatFloats + n % kBwdRows;
      lse[m] = st[kStatLse] * c;
      del[m] = st[kStatDelta];
    }
  }
  const int2 range = split_keys(rt.row0 < qlen ? keys.len : 0, pc.piece, pc.pieces, kTileKeys);
  const int turns = tiles_of(range.y - range.x, kTileKeys);
  KeyCopies<kMasked> copy;
  copy.begin(A.k, A.v, b, hk, keys, range.x, turns, wave, lane);
  auto place = [&](int i) __attribute__((always_inline)) { return lds_address(&lds[i % kRing][0][0]); };

  struct Scores {
    f32x16 s[2], x[2];  // scores, then P; X
  } sa, sb;
  f32x16 dq[2][4] = {};
  bf16x8 ring[kHold];
  uint32_t pw[2][8];  // dS, but for the factor scale
  const RowPlace rp = row_place(lane);
  const int cp = col_place(lane);
  // the fragment of slots 2 f and 2 f + 1 of a turn on tile `now` whose products read tile `then`
  auto fragment = [&](int f, const uint8_t* now, const uint8_t* then) __attribute__((always_inline)) {
    if (f < 8) return row_frag(now, rp, f);
    if (f < 16) return row_frag(now + kTile32, rp, f - 8);
    return col_frag(then + cp, (f - 16) >> 2, f & 3);
  };
  auto finish = [&](const Scores& old, int m, int r) __attribute__((always_inline)) {  // keys r, r + 1
    pw[m][r >> 1] = pack_bf16x2(old.s[m][r] * (old.x[m][r] + del[m]), old.s[m][r + 1] * (old.x[m][r + 1] + del[m]));
    pin(pw[m][r >> 1]);
  };
  auto hold_operands = [&]() __attribute__((always_inline)) {
    hold_in_agprs(qf[0]);
    hold_in_agprs(qf[1]);
    hold_in_agprs(gf[0]);
    hold_in_agprs(gf[1]);
  };
  auto turn = [&](int i, Scores& now, Scores& old) __attribute__((always_inline)) {
    constexpr int kSlots = 48;
    const uint8_t* tn = &lds[i % kRing][0][0];
    const uint8_t* to = &lds[(i + kRing - 1) % kRing][0][0];
    const uint8_t* next = &lds[(i + 1) % kRing][0][0];
#pragma unroll
    for (int d = 0; d < 4; ++d) asm volatile("" : "+a"(dq[0][d]), "+a"(dq[1][d]));
    hold_operands();
    each<0, kSlots>([&](auto slot) __attribute__((always_inline)) {
      constexpr int j = slot.value, f = j / 2, m = j & 1;
      if constexpr (j == kSlots - 14) {
        copies_landed<0>();
        copy.start(place(i + 2), place(i + 2) + kTile32);
        slot_end();
      }
      if constexpr (j >= kSlots - 13 && j < kSlots - 9) copy.part(j - (kSlots - 13));
      const bf16x8 a = ring[f % kHold];
      if constexpr (j < 16) {
        if constexpr (j < 2) score_first_a(now.s[m], a, qf[m][f]);
        else score_a(now.s[m], a, qf[m][f]);
      } else if constexpr (j < 32) {
        if constexpr (j < 18) score_first_a(now.x[m], a, gf[m][f - 8]);
        else score_a(now.x[m], a, gf[m][f - 8]);
      } else {
        constexpr int d = f & 3, y = (f - 16) >> 2;
        const uint4 w = make_uint4(pw[m][4 * y], pw[m][4 * y + 1], pw[m][4 * y + 2], pw[m][4 * y + 3]);
        dq[m][d] = mfma(a, __builtin_bit_cast(bf16x8, w), dq[m][d]);
      }
      if constexpr (m == 0) {
        constexpr int g = f + kAhead;
        ring[g % kHold] = g < kSlots / 2 ? fragment(g, tn, to) : fragment(g - kSlots / 2, next, tn);
      }
      if constexpr (j < 32 && j % 2 == 0) finish(old, (j >> 1) & 1, (j >> 2) * 2);
      if constexpr (j >= 18) {  // the exponentials: 32 in 30 slots
#pragma unroll
        for (int e = (j - 18) * 16 / 15; e < (j - 17) * 16 / 15; ++e) {
          float p = __builtin_amdgcn_exp2f(__builtin_fmaf(now.s[e & 1][e >> 1], c, lse[e & 1]));
          pin(p);
          now.s[e & 1][e >> 1] = p;
        }
      }
      slot_end();
    });
    const int key = range.x + i * kTileKeys;
    if (key + kTileKeys > keys.len || i >= turns) {
      const int to_key = i < turns ? keys.len : 0;  // (past the last tile: none)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (key + 4 * hh + 8 * (r >> 2) + (r & 3) >= to_key) now.s[0][r] = now.s[1][r] = 0.0f;
    }
  };
  if (turns > 0) {
    copy.all(place(0), place(0) + kTile32);
#pragma unroll
    for (int n = 0; n < 4; ++n) {  // turn 0's products, of dS = 0, take the same
      copy.to_k += n ? 0 : place(kRing - 1) - place(0);
      copy.to_v += n ? 0 : place(kRing - 1) - place(0);
      copy.part(n);
    }
    copies_landed<0>();
    hold_operands();
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      pin(lse[m]);
      pin(del[m]);
    }
    all_landed();
    copy.all(place(1), place(1) + kTile32);
    sb = Scores{};
#pragma unroll
    for (int f = 0; f < kAhead; ++f) ring[f] = fragment(f, &lds[0][0][0], nullptr);
    for (int i = 0; i <= turns; i += 2) {
      turn(i, sa, sb);
      turn(i + 1, sb, sa);
    }
    copies_landed<0>();  // none is under way when the wave ends
  }
  const int first = rt.row0 + 64 * wave;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    if (pc.pieces > 1) {
      float* o = A.dq_parts +
                 (((int64_t)(pc.tile - A.plan.full) * pc.pieces + pc.piece) * kCrossRows + row + 32 * m - rt.row0) * D + 4 * hh;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(o + 32 * d + 8 * q) =
              make_float4(dq[m][d][4 * q], dq[m][d][4 * q + 1], dq[m][d][4 * q + 2], dq[m][d][4 * q + 3]);
    } else {  // zero behind the sequence
      const bool valid = row + 32 * m < qlen;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) dq[m][d][r] = valid ? dq[m][d][r] * s.scale : 0.0f;
      store_rows(reinterpret_cast<uint8_t*>(lds) + wave * kOutBytes, lane,
                 A.dq.p + b * A.dq.sb + h * A.dq.sh + (int64_t)(first + 32 * m) * A.dq.sn, A.dq.sn, 0, s.N - first - 32 * m,
                 [&](int d, int q) { return pack4(dq[m][d], q); });
    }
  }
}

// A wave's 32 rows (of keys) to the rows of memory that order[i] names, i < rows.
template <class Words>
__device__ __forceinline__ void store_ordered(uint8_t* mine, int lane, uint16_t* to, int64_t sn, const int32_t* order,
                                              int rows, Words&& words) {
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
    if (r < rows) *reinterpret_cast<uint4*>(to + (int64_t)order[r] * sn + 8 * cc) = x;
  }
  asm volatile("" ::: "memory");
}

// dk, dv of 128 keys of one key head, 32 keys a wave, over the rows of every head of
// its group or of a piece of them (so a shared head's gradient is summed in registers,
// heads in order).
template <bool kMasked>
__device__ __forceinline__ void dkv_of(const CrossBwd& A, uint8_t (*lds)[2][kTile32], float (*stat)[kStatFloats], int wg,
                                       int wgs) {
  constexpr int kAhead = 8;
  // lds: q, dout
  const CrossShape& s = A.s;
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  const int tiles = tiles_of(s.M, kCrossKeys), pieces = A.head_pieces * A.row_pieces;
  const int id = xcd_local_id(wg, wgs), at = id / pieces;
  const int2 bh = slab_of(at / tiles, s.Hk, s);
  const int piece = id % pieces, row_piece = piece % A.row_pieces;
  const int hk = bh.y, b = bh.x, tile = at % tiles;
  const int qlen = query_len(s, b);
  const Keys<kMasked> keys(s, A.order, A.counts, b);
  const int per = s.H / s.Hk / A.head_pieces, h0 = (hk * A.head_pieces + piece / A.row_pieces) * per;  // the piece's heads
  const int key0 = tile * kCrossKeys, key = key0 + 32 * wave + l32;
  const bool valid = key < keys.len;
  const float c = s.scale * kLog2e;

  bf16x8 kf[8], vf[8];
  const int64_t key_row = valid ? keys.at(key) : 0;
  load_row(kf, A.k.p + b * A.k.sb + hk * A.k.sh + key_row * A.k.sn, valid, hh);
  load_row(vf, A.v.p + b * A.v.sb + hk * A.v.sh + key_row * A.v.sn, valid, hh);

  // the tiles of rows, head after head
  const int row_tiles = tiles_of(s.N, kBwdRows);
  const int all = key0 < keys.len ? tiles_of(qlen, kBwdRows) : 0;
  const int first = (int)((int64_t)all * row_piece / A.row_pieces);
  const int end = (int)((int64_t)all * (row_piece + 1) / A.row_pieces);
  const int head_turns = end - first, turns = head_turns * per;

  const uint32_t at0 = lds_address(&lds[0][0][0]) + wave * kRowBlock;
  const uint32_t stat0 = lds_address(&stat[0][0]);
  const int copy_row = 8 * wave + (lane >> 3);
  const uint16_t* qh = A.q.p + b * A.q.sb + (int64_t)h0 * A.q.sh;
  const uint16_t* gh = A.dout.p + b * A.dout.sb + (int64_t)h0 * A.dout.sh;
  const float* sth = A.stats + (int64_t)(b * s.H + h0) * row_tiles * kStatFloats;
  // Tile after tile (head after head) into the ring, one kilobyte at a time; past
  // the last tile it comes again, and is not used.
  constexpr int kCopies = 5;
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
      cp_.q = qh + cp_.u * A.q.sh + (int64_t)first * kBwdRows * A.q.sn;
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
    cp_.to = __builtin_amdgcn_readfirstlane(at0 + (place % kRing) * (2 * kTile32));
    cp_.to_st = __builtin_amdgcn_readfirstlane(stat0 + (place % kRing) * (kStatFloats * 4));
    if (cp_.t + 1 == end) {  // rows past the sequence: its last row again (their P is 0)
      const int r = min(copy_row, qlen - 1 - cp_.t * kBwdRows);
      cp_.oq = copy_offset(r, A.q.sn, lane);
      cp_.og = copy_offset(r, A.dout.sn, lane);
    }
  };
  auto copy_part = [&](int n) __attribute__((always_inline)) {
    if (n == 4) copy_256(cp_.to_st, cp_.st, lane * 4);
    else copy_1k(cp_.to + n / 2 * kTile32 + n % 2 * 1024, n / 2 ? cp_.g : cp_.q, (n / 2 ? cp_.og : cp_.oq) + n % 2 * 128);
  };
  auto copy = [&](int i, int place) __attribute__((always_inline)) {
    copy_start(i, place);
#pragma unroll
    for (int n = 0; n < kCopies; ++n) copy_part(n);
  };

  struct Scores {
    f32x16 s, x;  // scores, X - delta
    float p[16];
  } sa, sb;
  f32x16 dv[4] = {}, dk[4] = {};
  bf16x8 ring[kAhead];
  uint32_t pw[2][8];  // P, dS
  const RowPlace rp = row_place(lane);
  const int cp = col_place(lane);
  auto hold_operands = [&]() __attribute__((always_inline)) {
    hold_in_agprs(kf);
    hold_in_agprs(vf);
  };
  auto fragment = [&](int i, const uint8_t* now, const uint8_t* then) __attribute__((always_inline)) {
    if (i < 8) return row_frag(now, rp, i);
    if (i < 16) return row_frag(now + kTile32, rp, i - 8);
    const int j = i - 16;  // y, d, which: dv, dk
    return col_frag(then + (j % 2 ? 0 : kTile32) + cp, j >> 3, (j >> 1) & 3);
  };
  // rows 4 q .. 4 q + 3 of a lane's sixteen
  auto put = [&](f32x16& x, int q, const float* st) __attribute__((always_inline)) {
    const float4 f = *reinterpret_cast<const float4*>(st + 8 * q + 4 * hh);
    x[4 * q] = f.x;
    x[4 * q + 1] = f.y;
    x[4 * q + 2] = f.z;
    x[4 * q + 3] = f.w;
  };
  // P and dS of rows r, r + 1 of a lane's sixteen of the last tile
  auto finish = [&](const Scores& old, int r) __attribute__((always_inline)) {
    pw[0][r >> 1] = pack_bf16x2(old.p[r], old.p[r + 1]);
    pw[1][r >> 1] = pack_bf16x2(old.p[r] * old.x[r], old.p[r + 1] * old.x[r + 1]);
    pin(pw[0][r >> 1]);
    pin(pw[1][r >> 1]);
  };
  auto turn = [&](int i, Scores& now, Scores& old) __attribute__((always_inline)) {
    constexpr int kSlots = 32;
    const uint8_t* tn = &lds[i % kRing][0][0];
    const uint8_t* to = &lds[(i + kRing - 1) % kRing][0][0];
    const uint8_t* next = &lds[(i + 1) % kRing][0][0];
    const float* stn = stat[i % kRing];
    const float* next_st = stat[(i + 1) % kRing];
    // (the gradients where only MFMAs reach them)
#pragma unroll
    for (int d = 0; d < 4; ++d) asm volatile("" : "+a"(dv[d]), "+a"(dk[d]));
    hold_operands();
    each<0, kSlots>([&](auto slot) __attribute__((always_inline)) {
      constexpr int j = slot.value;
      if constexpr (j == kSlots - 8) {
        copies_landed<0>();
        copy_start(i + 2, i + 2);
        slot_end();
      }
      if constexpr (j >= kSlots - 7 && j < kSlots - 7 + kCopies) copy_part(j - (kSlots - 7));
      const bf16x8 f = ring[j % kAhead];
      if constexpr (j < 8) {
        score_a(now.s, f, kf[j]);
      } else if constexpr (j < 16) {
        score_a(now.x, f, vf[j - 8]);
      } else {
        constexpr int w = j % 2, d = ((j - 16) >> 1) & 3, y = (j - 16) >> 3;
        const bf16x8 p = __builtin_bit_cast(bf16x8, make_uint4(pw[w][4 * y], pw[w][4 * y + 1], pw[w][4 * y + 2], pw[w][4 * y + 3]));
        if constexpr (w == 0) dv[d] = mfma(f, p, dv[d]);
        else dk[d] = mfma(f, p, dk[d]);
      }
      constexpr int k = j + kAhead;
      ring[j % kAhead] = k < kSlots ? fragment(k, tn, to) : fragment(k - kSlots, next, tn);
      if constexpr (j < 16 && j % 2 == 0) finish(old, j);
      if constexpr (j < 4) put(now.x, j, stn + kStatDelta);
      // the next turn's scores start from the rows' log sums
      if constexpr (j >= 24 && j < 28) put(old.s, j - 24, next_st + kStatLse);
      if constexpr (j >= 10) {  // the exponentials: 16 in 22 slots
#pragma unroll
        for (int e = (j - 10) * 8 / 11; e < (j - 9) * 8 / 11; ++e) {
          now.p[e] = __builtin_amdgcn_exp2f(now.s[e] * c);
          pin(now.p[e]);
        }
      }
      slot_end();
    });
    if (key0 + 32 * wave + 32 > keys.len || i >= turns) {
      if (!valid || i >= turns) {  // (past the last tile: none)
#pragma unroll
        for (int r = 0; r < 16; ++r) now.p[r] = 0.0f;
      }
    }
  };
  if (turns > 0) {
    copy(0, 0);
    copy(0, kRing - 1);  // turn 0's products, of P = dS = 0
    copies_landed<0>();
    hold_operands();
    all_landed();
    copy(1, 1);
    sb = Scores{};
#pragma unroll
    for (int q = 0; q < 4; ++q) put(sa.s, q, stat[0] + kStatLse);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) ring[j] = fragment(j, &lds[0][0][0], nullptr);
    for (int i = 0; i <= turns; i += 2) {
      turn(i, sa, sb);
      turn(i + 1, sb, sa);
    }
    copies_landed<0>();  // none is under way when the wave ends
  }
  if (pieces > 1) {
    float* o = A.dkv_parts + (((int64_t)at * pieces + piece) * 2 * kCrossKeys + key - key0) * D + 4 * hh;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x16& x = m ? dk[d] : dv[d];
          *reinterpret_cast<float4*>(o + m * kCrossKeys * D + 32 * d + 8 * q) =
              make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
        }
    return;
  }
  // zero where a key is not visible
  uint8_t* mine = reinterpret_cast<uint8_t*>(lds) + wave * kOutBytes;
  const int first_key = key0 + 32 * wave;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    f32x16(&x)[4] = m ? dk : dv;
    const Rows& y = m ? A.dk : A.dv;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[d][r] = valid ? x[d][r] * (m ? s.scale : 1.0f) : 0.0f;
    uint16_t* base = y.p + b * y.sb + hk * y.sh;
    auto words = [&](int d, int q) { return pack4(x[d], q); };
    if (kMasked) store_ordered(mine, lane, base, y.sn, keys.order + first_key, s.M - first_key, words);
    else store_rows(mine, lane, base + (int64_t)first_key * y.sn, y.sn, 0, s.M - first_key, words);
  }
}

// Both in one launch, the keys' workgroups first: what either leaves of the last
// round of the chip's 256 CUs the other fills.
template <bool kMasked>
__global__ __launch_bounds__(256, 1) void cross_bwd_kernel(CrossBwd A, int key_wgs) {
  struct Lds {
    uint8_t tiles[kRing][2][kTile32];
    float stat[kRing][kStatFloats];
  };
  __shared__ __attribute__((aligned(1024))) Lds lds;
  lds_poison(&lds, sizeof(lds));
  lds_poison_done();
  if ((int)blockIdx.x < key_wgs)
    dkv_of<kMasked>(A, lds.tiles, lds.stat, blockIdx.x, key_wgs);
  else
    dq_of<kMasked>(A, lds.tiles, blockIdx.x - key_wgs);
}

// Few keys (kShortBwdKeys at most): one workgroup has all of a key head's, 32 a wave, and
// takes blocks of 32 rows of its heads, every parts-th one, so that a row is read once and
// the five products are five (the walks above, which meet the rows twice, take seven).  A
// wave finds S and X of its keys as Q K^T and dout V^T, whose registers are the operands of
// dv and dk; dS goes through LDS, where every wave takes all the keys' for dq of 32 dims.
// delta is found from the rows once they are in LDS, the next block's bytes in flight.
//
// 24 heads of 12,480 rows over 77 keys 137 us, 40 of 111,600 1,594 (3.6 TB/s of rows), the
// walks 176 and 2,153.  What bounds it is a block's chain of products in one wave a SIMD, 3
// us: with all its bytes sent for two blocks ahead, straight into LDS, 158 and 1,843; with
// the rows through registers, which the compiler moves between files, 150 and 1,738.
constexpr int kShortBwdKeys = kCrossKeys;
__global__ __launch_bounds__(256, 1) void cross_short_bwd_kernel(CrossBwd A) {
  struct Lds {
    uint8_t rows[2][2][kTile32];  // q and dout of a block and the next
    uint8_t ds[4][kTile32];          // dS of a wave's keys, a key's 32 rows at the start of its 256 bytes; K to begin with
    uint8_t dq[kOutBytes];           // the last block's dq, on its way out
    float lse[kBwdRows], delta[kBwdRows];  // -log2 of the rows' sums (-inf: P is 0); -delta
  };
  __shared__ __attribute__((aligned(1024))) Lds lds;
  lds_poison(&lds, sizeof(lds));
  lds_poison_done();
  const CrossShape& s = A.s;
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  const int parts = A.row_pieces, slab = blockIdx.x / parts, part = blockIdx.x % parts;
  const int2 bh = slab_of(slab, s.Hk, s);
  const int b = bh.x, hk = bh.y, per = s.H / s.Hk;
  const int qlen = query_len(s, b), klen = key_len(s, b);
  const float c = s.scale * kLog2e;
  const RowPlace rp = row_place(lane);
  const int cp = col_place(lane);

  // the keys: rows of K and V in registers as the scores take them, and 32 dims of all of K
  const uint16_t* k = A.k.p + b * A.k.sb + hk * A.k.sh;
  const int r16 = t >> 4, cc = t & 15;  // of 16 threads a row
  const int own0 = 8 * wave + (lane >> 4);  // of the block's rows this thread has chunk cc of this one and the fourth after
  auto place = [&](int row) __attribute__((always_inline)) {  // of chunk cc of a tile's row
    return (row >> 3) * kRowBlock + (cc >> 3) * 1024 + (row & 7) * 128 + ((cc & 7) ^ swizzle(row & 7)) * 16;
  };
  auto seen = [&](int key) __attribute__((always_inline)) {
    return key < klen && (!s.mask || s.mask[(int64_t)b * s.M + key] != 0);
  };
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const int key = 16 * u + r16;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (seen(key)) x = *reinterpret_cast<const uint4*>(k + (int64_t)key * A.k.sn + 8 * cc);
    *reinterpret_cast<uint4*>(lds.ds[u >> 1] + place(16 * (u & 1) + r16)) = x;
  }
  const int key = 32 * wave + l32;
  const bool valid = seen(key), any = __any(valid) != 0, all = __all(valid) != 0;
  bf16x8 kf[8], vf[8], kt[8];
  load_row(vf, A.v.p + b * A.v.sb + hk * A.v.sh + (int64_t)key * A.v.sn, valid, hh);
  __syncthreads();
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) {
    kf[kk] = row_frag(lds.ds[wave], rp, kk);
    kt[kk] = col_frag(lds.ds[kk >> 1] + cp, kk & 1, wave);
  }
  f32x16 dv[4] = {}, dk[4] = {};

  // the blocks that have rows; those that have none get zeros
  const int with_rows = tiles_of(qlen, kBwdRows), blocks = per * with_rows, none = per * (tiles_of(s.N, kBwdRows) - with_rows);
  for (int i = part; i < none; i += parts) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int n = (with_rows + i / per) * kBwdRows + r16 + 16 * u;
      if (n < s.N)
        *reinterpret_cast<uint4*>(A.dq.p + b * A.dq.sb + (hk * per + i % per) * A.dq.sh + (int64_t)n * A.dq.sn + 8 * cc) =
            make_uint4(0, 0, 0, 0);
    }
  }
  struct Block {
    int h, row0;
  };
  auto block = [&](int i) __attribute__((always_inline)) {
    const int u = i / with_rows;
    return Block{hk * per + u, (i - u * with_rows) * kBwdRows};
  };
  // Rows of block x on their way, those behind the sequence as its last one (their P is 0):
  // q and dout into LDS, a wave eight of them; of out, what it left and the log sums a
  // thread its own rows.
  uint4 xo[2], xl[2];
  float xs[2];
  auto load = [&](const Block& x, int to) __attribute__((always_inline)) {
    const int64_t row0 = ((int64_t)b * s.H + x.h) * s.N;
    const int last = qlen - 1 - x.row0, copied = min(8 * wave + (lane >> 3), last);
    const uint16_t* q = A.q.p + b * A.q.sb + x.h * A.q.sh + (int64_t)x.row0 * A.q.sn;
    const uint16_t* g = A.dout.p + b * A.dout.sb + x.h * A.dout.sh + (int64_t)x.row0 * A.dout.sn;
    const uint32_t at = __builtin_amdgcn_readfirstlane(lds_address(&lds.rows[0][0][0]) + to * 2 * kTile32 + wave * kRowBlock);
    const uint32_t oq = copy_offset(copied, A.q.sn, lane), og = copy_offset(copied, A.dout.sn, lane);
    copy_1k(at, q, oq);
    copy_1k(at + 1024, q, oq + 128);
    copy_1k(at + kTile32, g, og);
    copy_1k(at + kTile32 + 1024, g, og + 128);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int n = x.row0 + min(own0 + 4 * u, last);
      xo[u] = *reinterpret_cast<const uint4*>(A.out.p + b * A.out.sb + x.h * A.out.sh + (int64_t)n * A.out.sn + 8 * cc);
      xl[u] = *reinterpret_cast<const uint4*>(A.left + (row0 + n) * D + 8 * cc);
      xs[u] = A.lse[row0 + n];
    }
  };
  // dq of block x, which all waves have left in LDS, to memory
  auto flush = [&](const Block& x) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = own0 + 4 * u, n = x.row0 + r;
      uint4 y = *reinterpret_cast<const uint4*>(lds.dq + r * kOutStride + 16 * cc);
      if (n >= qlen) y = make_uint4(0, 0, 0, 0);
      if (n < s.N) *reinterpret_cast<uint4*>(A.dq.p + b * A.dq.sb + x.h * A.dq.sh + (int64_t)n * A.dq.sn + 8 * cc) = y;
    }
  };

  if (part < blocks) load(block(part), 0);
  int now = 0;
  for (int i = part; i < blocks; i += parts, now ^= 1) {
    const Block at = block(i);
    const uint8_t *tq = lds.rows[now][0], *tg = lds.rows[now][1];
    // (what only MFMAs reach, where the rows on their way need no room)
#pragma unroll
    for (int d = 0; d < 4; ++d) asm volatile("" : "+a"(dv[d]), "+a"(dk[d]));
    hold_in_agprs(kt);
    copies_landed<0>();  // this wave's rows
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = own0 + 4 * u;
      float o[8], g[8], left[8], d = 0.0f;
      unpack_bf16x8(xo[u], o);
      unpack_bf16x8(*reinterpret_cast<const uint4*>(tg + place(r)), g);
      unpack_bf16x8(xl[u], left);
#pragma unroll
      for (int e = 0; e < 8; ++e) d = __builtin_fmaf(g[e], o[e] + left[e], d);
      d = row_sumsq_lanes16(d);
      if (cc == 0) {
        const bool some = at.row0 + r < qlen && xs[u] > -3e38f;
        lds.lse[r] = some ? -xs[u] * kLog2e : -__builtin_inff();
        lds.delta[r] = some ? -d : 0.0f;
      }
    }
    __syncthreads();
    load(block(i + parts < blocks ? i + parts : i), now ^ 1);  // (the last one again is not used)
    if (i != part) flush(block(i - parts));
    if (any) {
      f32x16 sc, x;
      hold_in_agprs(kf);
      hold_in_agprs(vf);
      score_first_a(sc, row_frag(tq, rp, 0), kf[0]);
      score_first_a(x, row_frag(tg, rp, 0), vf[0]);
#pragma unroll
      for (int kk = 1; kk < 8; ++kk) {
        score_a(sc, row_frag(tq, rp, kk), kf[kk]);
        score_a(x, row_frag(tg, rp, kk), vf[kk]);
      }
      settle(sc, x);
      uint32_t pw[2][8];
#pragma unroll
      for (int g = 0; g < 4; ++g) {  // rows 8 g + 4 hh on
        const float4 l = *reinterpret_cast<const float4*>(lds.lse + 8 * g + 4 * hh);
        const float4 e = *reinterpret_cast<const float4*>(lds.delta + 8 * g + 4 * hh);
        float p[4] = {__builtin_fmaf(sc[4 * g], c, l.x), __builtin_fmaf(sc[4 * g + 1], c, l.y),
                      __builtin_fmaf(sc[4 * g + 2], c, l.z), __builtin_fmaf(sc[4 * g + 3], c, l.w)};
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          p[z] = __builtin_amdgcn_exp2f(p[z]);
          if (!all) p[z] = valid ? p[z] : 0.0f;
        }
        pw[0][2 * g] = pack_bf16x2(p[0], p[1]);
        pw[0][2 * g + 1] = pack_bf16x2(p[2], p[3]);
        pw[1][2 * g] = pack_bf16x2(p[0] * (x[4 * g] + e.x), p[1] * (x[4 * g + 1] + e.y));
        pw[1][2 * g + 1] = pack_bf16x2(p[2] * (x[4 * g + 2] + e.z), p[3] * (x[4 * g + 3] + e.w));
        *reinterpret_cast<uint2*>(lds.ds[wave] + (l32 >> 3) * kRowBlock + (l32 & 7) * 128 + (g ^ swizzle(l32 & 7)) * 16 + 8 * hh) =
            make_uint2(pw[1][2 * g], pw[1][2 * g + 1]);
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const bf16x8 p = __builtin_bit_cast(bf16x8, make_uint4(pw[0][4 * y], pw[0][4 * y + 1], pw[0][4 * y + 2], pw[0][4 * y + 3]));
        const bf16x8 ds = __builtin_bit_cast(bf16x8, make_uint4(pw[1][4 * y], pw[1][4 * y + 1], pw[1][4 * y + 2], pw[1][4 * y + 3]));
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          dv[d] = mfma(col_frag(tg + cp, y, d), p, dv[d]);
          dk[d] = mfma(col_frag(tq + cp, y, d), ds, dk[d]);
        }
      }
    }
    __syncthreads();
    f32x16 dq = {};
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (32 * u < klen) {
#pragma unroll
        for (int y = 0; y < 2; ++y) dq = mfma(kt[2 * u + y], col_frag(lds.ds[u] + cp, y, 0), dq);
      }
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<uint2*>(lds.dq + l32 * kOutStride + 64 * wave + 16 * g + 8 * hh) =
          make_uint2(pack_bf16x2(dq[4 * g] * s.scale, dq[4 * g + 1] * s.scale),
                     pack_bf16x2(dq[4 * g + 2] * s.scale, dq[4 * g + 3] * s.scale));
  }
  all_landed();  // none is under way when the wave ends
  __syncthreads();
  if (part < blocks) flush(block(part + (blocks - 1 - part) / parts * parts));
  __syncthreads();
  if (32 * wave >= s.M) return;
  // zero where a key is not visible
  if (parts > 1) {
    float* o = A.dkv_parts + (((int64_t)slab * parts + part) * 2 * kCrossKeys + key) * D + 4 * hh;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x16& x = m ? dk[d] : dv[d];
          *reinterpret_cast<float4*>(o + m * kCrossKeys * D + 32 * d + 8 * g) =
              valid ? make_float4(x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
    return;
  }
  uint8_t* mine = reinterpret_cast<uint8_t*>(&lds) + wave * kOutBytes;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    f32x16(&x)[4] = m ? dk : dv;
    const Rows& y = m ? A.dk : A.dv;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[d][i] = valid ? x[d][i] * (m ? s.scale : 1.0f) : 0.0f;
    store_rows(mine, lane, y.p + b * y.sb + hk * y.sh + (int64_t)(32 * wave) * y.sn, y.sn, 0, s.M - 32 * wave,
               [&](int d, int g) { return pack4(x[d], g); });
  }
}

// dq of a tile that was cut, the pieces summed in order, 16 rows a workgroup; then dv
// and dk of key tiles that were, 16 rows of one of them.
constexpr int kJoinRows = 16;
template <bool kMasked>
__global__ __launch_bounds__(256) void cross_end_kernel(CrossBwd A) {
  const CrossShape& s = A.s;
  const int64_t cut = row_tiles_of(s) - A.plan.full;
  const int dq_blocks = (int)(cut * (kCrossRows / kJoinRows));
  const int r16 = threadIdx.x >> 4, cc = threadIdx.x & 15;
  auto sum = [&](float (&f)[8], const float* p, int pieces, int64_t step) __attribute__((always_inline)) {
#pragma unroll 4
    for (int u = 0; u < pieces; ++u) {
      const float4* at = reinterpret_cast<const float4*>(p + u * step + 8 * cc);
      const float4 x = at[0], y = at[1];
      f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
      f[4] += y.x; f[5] += y.y; f[6] += y.z; f[7] += y.w;
    }
  };
  float f[8] = {};
  if ((int)blockIdx.x >= dq_blocks) {
    const int tiles = tiles_of(s.M, kCrossKeys), per_tile = kCrossKeys / kJoinRows;
    const int w = blockIdx.x - dq_blocks, m = w & 1, id = (w >> 1) / per_tile;
    const int r = (w >> 1) % per_tile * kJoinRows + r16, key = id % tiles * kCrossKeys + r;
    const int2 bh = slab_of(id / tiles, s.Hk, s);
    if (key >= s.M) return;
    const Keys<kMasked> keys(s, A.order, A.counts, bh.x);
    const int pieces = A.head_pieces * A.row_pieces;
    if (key < keys.len)
      sum(f, A.dkv_parts + (((int64_t)id * pieces * 2 + m) * kCrossKeys + r) * D, pieces, (int64_t)2 * kCrossKeys * D);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= m ? s.scale : 1.0f;
    const Rows& y = m ? A.dk : A.dv;
    *reinterpret_cast<uint4*>(y.p + bh.x * y.sb + bh.y * y.sh + (int64_t)keys.at(key) * y.sn + 8 * cc) = pack_bf16x8(f);
    return;
  }
  const int tile = blockIdx.x / (kCrossRows / kJoinRows), r = blockIdx.x % (kCrossRows / kJoinRows) * kJoinRows + r16;
  const RowTile rt = row_tile(A.plan.full + tile, s);
  const int row = rt.row0 + r;
  if (row >= s.N) return;
  if (row < query_len(s, rt.b))
    sum(f, A.dq_parts + ((int64_t)tile * A.plan.pieces * kCrossRows + r) * D, A.plan.pieces, (int64_t)kCrossRows * D);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] *= s.scale;
  *reinterpret_cast<uint4*>(A.dq.p + rt.b * A.dq.sb + rt.h * A.dq.sh + (int64_t)row * A.dq.sn + 8 * cc) = pack_bf16x8(f);
}

}  // namespace

// A launch is a 1D grid of fewer than 2^32 threads.
static bool fits(int64_t workgroups, int threads) { return workgroups < ((int64_t)1 << 32) / threads; }
// Row tiles of a forward call that runs in line.
constexpr int64_t kMostTiles = 1 << 20;
static size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

CrossPlan cross_plan(const CrossShape& s, bool ragged) {
  CrossPlan p = {};
  const int64_t tiles = row_tiles_of(s), turns = tiles_of(s.M, kTileKeys);
  // Groups of 32 rows where they all stand on the chip at once, or hold all of a key
  // head's rows: 24 heads over 512 keys, 256 rows (192 groups) 13.0 us, in tiles 22.8; 384
  // rows (288) 23.9, 22.9; over 4,096 keys 41, 48 and 77, 53; 16 x 16 heads over 512, 32
  // rows (256) 17.8, 25.9, 64 rows (512) 26.4, 26.1.  (Over many more keys the groups,
  // which read a fragment for one MFMA where tiles read it for two, fall behind from fewer
  // rows on: 8 heads over 12,480 keys, 256 rows 41 us, in tiles 52; 512 65, 53; 1,024 104,
  // 71; over 30,000 72, 67; 130, 83; 236, 131.)
  p.few = few_groups(s) == 1 || (int64_t)s.B * s.Hk * few_groups(s) <= kCus;
  if (p.few) {
    // As many pieces as give every CU a workgroup, of 512 keys or more (one row of 24
    // heads over 512 keys 9.4 us in one piece, 13.2 in two, with the join; 4 x 8 heads
    // over 2,048 21.0, 16.7, 13.7 in four; 40 over 30,000 285, 110 in six).  Where lengths
    // differ two for every CU, of 1,024 or more: 32 caches of 256 to 8,192 keys, 8 heads,
    // 119 us in one piece, 103 in two, 113 in four; equal ones 183, 183, 187.
    const int64_t wgs = (int64_t)s.B * s.Hk * few_groups(s);
    int64_t n = std::min<int64_t>(kCus / wgs, s.M / 512);
    if (ragged && s.B > 1) n = std::max(n, std::min<int64_t>(2 * kCus / wgs, s.M / 1024));
    p.pieces = (int)(n < 1 ? 1 : n);
    return p;
  }
  p.pieces = 1;
  // Few keys: 24 heads of 12,480 rows over 77 45 us, over 256 53, for training 51 and 66;
  // in the ring 57, 70, 68 and 82.  64 x 24 heads of 300 rows over 200 127, 197.
  p.brief = s.M <= kShortKeys;
  p.workgroups = (int)std::min<int64_t>(kCus, p.brief ? tiles : tiles * turns);
  if (p.brief) return p;
  // What whole tiles leave idle, in turns of 0.9 us, against the shares' way through memory
  // (20 to 30 us), and against the clock, which rises where part of the chip idles: 24 heads
  // over 4,096 keys, 1,024 rows (80 turns idle) 111 us whole, 79 split, 12,480 rows (52, a
  // twelfth of all) 577, 604; 8 heads of 4,097 over 12,480 (183) 312, 224; 24 of 1,024 over
  // 2,048 (40) 62, 58, over 1,024 (20) 37, 47.
  const double all = (double)((tiles + kCus - 1) / kCus * turns), idle = all - (double)(tiles * turns) / kCus;
  // Lengths, which are not known here, change nothing: 2 x 8 heads of up to 4,000 rows over
  // 8,000 masked keys would gain (171, 148), 4 x 24 heads lose (528, 576).
  p.split = idle > 30 && 8 * idle > all && !(ragged && s.B > kMaxByLength);
  return p;
}

static int64_t few_workgroups(const CrossShape& s, int pieces) {
  return (int64_t)s.B * s.Hk * pieces * few_groups(s);
}
// The visible keys' order and counts.
static size_t order_bytes(const CrossShape& s) { return s.mask ? up256(((size_t)s.B * s.M + s.B) * sizeof(int32_t)) : 0; }
static void launch_order(const CrossShape& s, int32_t* order, int32_t* counts, hipStream_t stream) {
  hipLaunchKernelGGL(cross_order_kernel, dim3((unsigned)s.B), dim3(kOrderThreads), 0, stream, s, order, counts);
}

size_t cross_fwd_bytes(const CrossShape& s, CrossFwd* a, void* ws) {
  if (a) a->ws = static_cast<float*>(ws);
  // (the most, with lengths or without: few rows' pieces with them, tiles' shares without)
  const CrossPlan p = cross_plan(s, false);
  if (p.few) {
    const int pieces = std::max(p.pieces, cross_plan(s, true).pieces);
    if (!fits(few_workgroups(s, pieces), kFewThreads)) return kTooLarge;
    return pieces > 1 ? (size_t)s.B * s.H * s.N * pieces * (D + 2) * sizeof(float) : 0;
  }
  if (p.brief) return 0;
  // (shared tiles, which a launch of 16 rows a workgroup joins, are far fewer)
  if (row_tiles_of(s) > kMostTiles || (s.mask && !fits(s.B, kOrderThreads))) return kTooLarge;
  const size_t order = order_bytes(s);
  if (a) {
    a->order = static_cast<int32_t*>(ws);
    a->counts = a->order + (size_t)s.B * s.M;
    a->ws = reinterpret_cast<float*>(static_cast<char*>(ws) + order);
  }
  return order + (p.split ? (size_t)2 * p.workgroups * kShareFloats * sizeof(float) : 0);
}

hipError_t launch_cross_fwd(const CrossFwd& a, hipStream_t stream) {
  const CrossShape& s = a.s;
  const CrossPlan p = cross_plan(s, s.q_lens || s.kv_lens || s.mask);
  if (p.few) {
    const auto kernel = s.mask ? cross_few_kernel<true> : cross_few_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)few_workgroups(s, p.pieces)), dim3(kFewThreads), 0, stream, a, p.pieces);
    if (p.pieces > 1)
      hipLaunchKernelGGL(cross_join_kernel, dim3((unsigned)((int64_t)s.B * s.H * s.N)), dim3(256), 0, stream, a, p.pieces);
    return hipGetLastError();
  }
  if (p.brief) {
    const auto kernel = s.M <= 32   ? (a.lse ? cross_short_kernel<1, true> : cross_short_kernel<1, false>)
                        : s.M <= 64 ? (a.lse ? cross_short_kernel<2, true> : cross_short_kernel<2, false>)
                        : s.M <= 128 ? (a.lse ? cross_short_kernel<4, true> : cross_short_kernel<4, false>)
                                    : (a.lse ? cross_short_kernel<8, true> : cross_short_kernel<8, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.workgroups), dim3(kShortThreads), 0, stream, a);
    return hipGetLastError();
  }
  if (s.mask) launch_order(s, a.order, a.counts, stream);
  const auto kernel = s.mask ? (a.lse ? cross_fwd_kernel<true, true> : cross_fwd_kernel<true, false>)
                             : (a.lse ? cross_fwd_kernel<false, true> : cross_fwd_kernel<false, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)p.workgroups), dim3(256), 0, stream, a, p.split);
  if (p.split)
    hipLaunchKernelGGL(cross_shares_kernel, dim3((unsigned)(row_tiles_of(s) * (kCrossRows / 16))), dim3(256), 0, stream, a,
                       p.workgroups);
  return hipGetLastError();
}

// Tiles [full, tiles) cut along the keys, in pieces of 512 keys or more.
static DiffTiles cut_tiles(int64_t tiles, int64_t full, int64_t pieces, int M) {
  pieces = std::min<int64_t>({pieces, M / 512, 16});
  if (pieces < 2) return {(int)tiles, 1};
  return {(int)full, (int)pieces};
}
// Pieces of the last tiles, which leave part of the chip idle, that fill it.
static int64_t filling(int64_t tiles, int64_t full) { return tiles > full ? kCus / (tiles - full) : 1; }

// The backward launch: the keys' workgroups, then the rows'.  Times in slots of an
// MFMA: a key tile 32 a block of 32 rows, times the heads that share it; a row tile 48
// a block of 32 keys.
struct BwdCost {
  int64_t keys, key, row;  // key tiles; a key tile's time, a row tile's
  double fair;             // a CU's time for everything if nothing idled
};
static BwdCost bwd_cost(const CrossShape& s) {
  BwdCost c = {(int64_t)s.B * s.Hk * tiles_of(s.M, kCrossKeys), (int64_t)(s.H / s.Hk) * tiles_of(s.N, kBwdRows) * 32,
               (int64_t)tiles_of(s.M, kTileKeys) * 48, 0.0};
  c.fair = (double)(c.keys * c.key + row_tiles_of(s) * c.row) / kCus;
  return c;
}
// A key tile walks the rows of all the query heads that share it.  Where that takes
// longer than the chip needs for everything, its heads and then their rows (256 or
// more) go to several workgroups, if that saves more than their sums' way through the
// workspace costs: 24 heads of 12,480 rows on 4 key heads of 512 keys 1,648 us whole, 343
// in pieces; on 24 381, 367; 8 heads of 4,097 rows over 12,480 keys 801, 735; 16 of 1,024
// over 1,024 51, 47.
struct KeyPieces {
  int heads, rows;
  int all() const { return heads * rows; }
};
static KeyPieces key_pieces(const CrossShape& s) {
  const BwdCost c = bwd_cost(s);
  const int per = s.H / s.Hk;
  KeyPieces least = {1, 1};
  double time = std::max((double)c.key, c.fair);
  auto consider = [&](KeyPieces p) {
    const double t = std::max((double)c.key / p.all(), c.fair) + 600 + 4.0 * c.keys * p.all();
    if (t < time) {
      time = t;
      least = p;
    }
  };
  for (int p = 2; p <= std::min(per, kCus); ++p)
    if (per % p == 0) consider({p, 1});
  for (int p = 2; p <= std::min(64, s.N / 256); ++p) consider({per, p});
  return least;
}
static DiffTiles bwd_tiles(const CrossShape& s, int pieces) {
  const int64_t tiles = row_tiles_of(s);
  const BwdCost c = bwd_cost(s);
  const int64_t keys = c.keys * pieces, key_cost = c.key / pieces;
  if (keys + tiles <= kCus) {
    // The chip has room for all: rows are cut (in pieces of 128 keys or more) where that
    // ends sooner, a start and the join taking some six turns each; past one round the
    // workgroups' mean and half of a last one.  (4 x 3 heads of 6 rows over 1,021 keys 43 us
    // whole, 24 cut; 3 x 4 on 2 of 274 over 4,375 142, 58; 8 of 512 over 512 31, 29.)
    constexpr double kStart = 6 * 48;
    int least = 1;
    double time = (double)std::max(key_cost, c.row) + kStart;
    for (int n = 2; n <= std::min(32, s.M / 128); ++n) {
      const double piece = (double)c.row / n;
      const double t = kStart + (keys + tiles * n <= kCus ? std::max((double)key_cost, piece) + kStart
                                                          : (keys * (key_cost + kStart) + tiles * n * (piece + kStart)) / kCus +
                                                                (piece + kStart) / 2);
      if (t < time) {
        time = t;
        least = n;
      }
    }
    return least > 1 ? DiffTiles{0, least} : DiffTiles{(int)tiles, 1};
  }
  const int64_t best = (keys * key_cost + tiles * c.row) / kCus;
  const int64_t round = keys / kCus, more = keys % kCus;  // `more` CUs take round + 1 key tiles
  const int64_t a = best - round * key_cost, b = a - key_cost;
  const int64_t full = std::min(tiles, (kCus - more) * (a > 0 ? a / c.row : 0) + more * (b > 0 ? b / c.row : 0));
  // what is left goes to the CUs' remaining time (2 x 8 heads of 300 rows over 4,000 keys 161
  // us whole, 75 cut; 8 of 2,048 over 2,048 81, 78)
  return cut_tiles(tiles, full, filling(tiles, full), s.M);
}

// Workgroups of the backward launches: the rows' statistics, both walks (the keys'
// first), the end (0: none is needed).
struct BwdGrids {
  int64_t stats, keys, walks, end;
};
static BwdGrids bwd_grids(const CrossShape& s, const KeyPieces& pieces, const DiffTiles& plan) {
  const int64_t key_tiles = bwd_cost(s).keys, rest = row_tiles_of(s) - plan.full;
  BwdGrids g;
  g.stats = (int64_t)s.B * s.H * tiles_of(s.N, kBwdRows);
  g.keys = key_tiles * pieces.all();
  g.walks = g.keys + plan.full + rest * plan.pieces;
  g.end = rest * (kCrossRows / kJoinRows);
  if (pieces.all() > 1) g.end += key_tiles * (kCrossKeys / kJoinRows) * 2;
  return g;
}

// Workgroups of a key head of few keys: as many as the chip has room for, of two blocks of
// rows or more, up to kMostParts, whose sums are joined.  Few key heads of many rows, which
// that would leave part of the chip idle with, walk as more keys do (one head of 20,000 rows
// over 77 keys 72 us in 32 parts, 32; 24 heads on 2 of 12,480 442, 170).
static int short_parts(const CrossShape& s) {
  const int64_t slabs = (int64_t)s.B * s.Hk, blocks = (int64_t)(s.H / s.Hk) * tiles_of(s.N, kBwdRows);
  constexpr int kMostParts = 32;
  if (s.M > kShortBwdKeys || (slabs * kMostParts < kCus && blocks > 2 * kMostParts)) return 0;
  return (int)std::max<int64_t>(1, std::min<int64_t>({kCus / slabs, blocks / 2, kMostParts}));
}

size_t cross_bwd_bytes(const CrossShape& s, CrossBwd* a, void* ws) {
  if (const int parts = short_parts(s)) {
    const int64_t slabs = (int64_t)s.B * s.Hk;
    if (a) {
      a->dkv_parts = static_cast<float*>(ws);
      a->plan = {(int)row_tiles_of(s), 1};
      a->head_pieces = 1;
      a->row_pieces = parts;
    }
    return parts > 1 ? (size_t)slabs * parts * 2 * kCrossKeys * D * sizeof(float) : 0;
  }
  const KeyPieces pieces = key_pieces(s);
  const DiffTiles plan = bwd_tiles(s, pieces.all());
  const BwdGrids g = bwd_grids(s, pieces, plan);
  if (!fits(g.stats, 16 * kBwdRows) || !fits(g.walks, 256) || !fits(g.end, 256) || (s.mask && !fits(s.B, kOrderThreads)))
    return kTooLarge;
  size_t at[4];
  at[0] = order_bytes(s);
  at[1] = at[0] + up256((size_t)g.stats * kStatFloats * sizeof(float));
  at[2] = at[1];
  if (plan.pieces > 1) at[2] += (size_t)(row_tiles_of(s) - plan.full) * plan.pieces * kCrossRows * D * sizeof(float);
  at[3] = at[2];
  if (pieces.all() > 1) at[3] += (size_t)bwd_cost(s).keys * pieces.all() * 2 * kCrossKeys * D * sizeof(float);
  if (a) {
    char* p = static_cast<char*>(ws);
    a->order = reinterpret_cast<int32_t*>(p);
    a->counts = a->order + (size_t)s.B * s.M;
    a->stats = reinterpret_cast<float*>(p + at[0]);
    a->dq_parts = reinterpret_cast<float*>(p + at[1]);
    a->dkv_parts = reinterpret_cast<float*>(p + at[2]);
    a->plan = plan;
    a->head_pieces = pieces.heads;
    a->row_pieces = pieces.rows;
  }
  return at[3];
}

hipError_t launch_cross_bwd(const CrossBwd& a, hipStream_t stream) {
  const CrossShape& s = a.s;
  const BwdGrids g = bwd_grids(s, {a.head_pieces, a.row_pieces}, a.plan);
  if (short_parts(s)) {
    hipLaunchKernelGGL(cross_short_bwd_kernel, dim3((unsigned)(s.B * s.Hk * a.row_pieces)), dim3(256), 0, stream, a);
    if (g.end) hipLaunchKernelGGL(cross_end_kernel<false>, dim3((unsigned)g.end), dim3(256), 0, stream, a);
    return hipGetLastError();
  }
  if (s.mask) launch_order(s, a.order, a.counts, stream);
  hipLaunchKernelGGL(cross_stats_kernel, dim3((unsigned)g.stats), dim3(16 * kBwdRows), 0, stream, a);
  const auto walk = s.mask ? cross_bwd_kernel<true> : cross_bwd_kernel<false>;
  hipLaunchKernelGGL(walk, dim3((unsigned)g.walks), dim3(256), 0, stream, a, (int)g.keys);
  if (g.end) {
    const auto end = s.mask ? cross_end_kernel<true> : cross_end_kernel<false>;
    hipLaunchKernelGGL(end, dim3((unsigned)g.end), dim3(256), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace sol
