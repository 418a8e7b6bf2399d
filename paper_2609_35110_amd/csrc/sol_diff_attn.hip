// Differential attention (sol_diff_attn_fwd, _bwd): for every output head the
// difference of two softmax maps over the same values,
//   out = softmax(scale q_0 k_0^T) v - lambda softmax(scale q_1 k_1^T) v,
// query heads 2h and 2h + 1 of q being the maps of output head h.
//
// One pass over the keys with the running maximum and sum of each row and map;
// scores S^T = K Q^T and outputs O^T = V^T P^T, so that a lane owns a row: its
// maximum, sum and rescaling are the lane's own, and P as the score MFMA
// leaves it is the operand of the next.  fp32 throughout but for the operands:
// P is rounded to bf16 (its row sum is not), as the values are bf16.
#include <hip/hip_runtime.h>

#include "sol_ops.h"
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

// The keys of split i of n: whole tiles, as even as they come.
__device__ __forceinline__ int2 split_keys(int klen, int i, int n, int tile) {
  const int tiles = (klen + tile - 1) / tile;
  const int per = (tiles + n - 1) / n;
  return make_int2(min(i * per * tile, klen), min((i + 1) * per * tile, klen));
}

// One map of 32 rows: a lane's row is lane % 32.
struct MapRows {
  f32x16 o[4];  // O^T: dims 32t + 8(r/4) + 4(lane/32) + r%4
  float m, l;   // maximum held to (raw scores), sum of this lane's half of the keys
};
__device__ __forceinline__ void clear(MapRows& x) {
#pragma unroll
  for (int t = 0; t < 4; ++t) x.o[t] = f32x16{};
  x.m = kNoMax;
  x.l = 0.0f;
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
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) x.o[t][r] *= keep;
    x.m = m;
  }
}

// P of 32 keys in place of their scores, and its sum.
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
  x.l += a + b;
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

// log2 of a row's sum of exponentials; -inf for a row without keys.
__device__ __forceinline__ float log2_sum(float m, float l, float c) {
  return l > 0.0f ? m * c + log2f(l) : -__builtin_inff();
}

// Partial results of split i of n: o fp32 [split][B][2H][N][128], then the
// log2 sums [split][B][2H][N].
struct Parts {
  float* o;
  float* l;
  int64_t rows;  // B 2H N
};
__device__ __forceinline__ Parts parts_of(float* ws, const DiffShape& s, int nsplit) {
  const int64_t rows = (int64_t)s.B * 2 * s.H * s.N;
  return {ws, ws + rows * nsplit * D, rows};
}

// ------------------------------------------------------------------- forward

// 128 rows of one head: waves 0..3 take 32 rows each of map 0, waves 4..7 the
// same rows of map 1, so that the two waves of a SIMD run one's exponentials
// under the other's MFMAs.  K and V tiles of 64 keys pass through LDS, two
// buffers, one barrier a tile.
template <bool kShared>
__global__ __launch_bounds__(512, 2) void diff_fwd_kernel(DiffFwd A, int nsplit) {
  constexpr int kTileElems = kDiffKeys * kStride;
  constexpr int kKTiles = kShared ? 1 : 2;
  __shared__ __attribute__((aligned(16))) uint16_t lds[2][(kKTiles + 1) * kTileElems];
  lds_poison(lds, sizeof(lds));
  lds_poison_done();
  const DiffShape& s = A.s;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  const int map = wave >> 2, group = wave & 3;
  const int tiles = (s.N + kDiffRows - 1) / kDiffRows;
  int id = xcd_local_id(blockIdx.x, gridDim.x);
  const int split = id % nsplit;
  id /= nsplit;
  const int tile = tiles - 1 - id % tiles;  // causal: the long rows first
  id /= tiles;
  const int h = id % s.H, b = id / s.H;
  const Seq sq = sequence(s, b);
  const int row0 = tile * kDiffRows;
  if (row0 >= sq.qlen) return;
  const int per = s.H / s.Hv, hv = h / per;
  const int row = row0 + 32 * group + l32;
  const bool valid = row < sq.qlen;
  const float c = s.scale * kLog2e;

  const uint16_t* k0 = A.k.p + b * A.k.sb + (kShared ? hv : 2 * hv) * A.k.sh;
  const uint16_t* k1 = k0 + (kShared ? 0 : A.k.sh);
  const uint16_t* v = A.v.p + b * A.v.sb + hv * A.v.sh;
  bf16x8 qf[8];
  load_row(qf, A.q.p + b * A.q.sb + (2 * h + map) * A.q.sh + (int64_t)row * A.q.sn, valid, hh);

  const int2 range = split_keys(sq.klen, split, nsplit, kDiffKeys);
  const int last = min(row + sq.shift, sq.klen - 1);  // of this lane's row
  const int last_row = min(row0 + kDiffRows, sq.qlen) - 1;
  const int kend = min(range.y, min(last_row + sq.shift, sq.klen - 1) + 1);
  // what every row of the wave sees, and what none does
  const int wave_row = row0 + 32 * group;
  const int all_to = min(wave_row + sq.shift, sq.klen - 1);
  const int none_from = wave_row < sq.qlen ? min(wave_row + 31 + sq.shift, sq.klen - 1) : -1;

  MapRows x;
  clear(x);
  const int tr = column_offset(lane);
  Stage<kDiffKeys, 512> sk0, sk1, sv;
  auto load = [&](int key) __attribute__((always_inline)) {
    sk0.load(k0, A.k.sn, key, kend, t);
    if (!kShared) sk1.load(k1, A.k.sn, key, kend, t);
    sv.load(v, A.v.sn, key, kend, t);
  };
  auto store = [&](int buf) __attribute__((always_inline)) {
    sk0.store(lds[buf], t);
    if (!kShared) sk1.store(lds[buf] + kTileElems, t);
    sv.store(lds[buf] + kKTiles * kTileElems, t);
  };
  if (range.x < kend) {
    load(range.x);
    store(0);
  }
  int buf = 0;
  for (int key = range.x; key < kend; key += kDiffKeys, buf ^= 1) {
    __syncthreads();
    const bool more = key + kDiffKeys < kend;
    if (more) load(key + kDiffKeys);
    if (key <= none_from) {
      const uint16_t* tk = lds[buf] + (kShared ? 0 : map * kTileElems);
      const uint16_t* tv = lds[buf] + kKTiles * kTileElems + tr;
      f32x16 sc[2] = {scores(tk, qf, lane), scores(tk + 32 * kStride, qf, lane)};
      if (key + kDiffKeys - 1 > all_to) {
        mask(sc[0], key + 4 * hh, last);
        mask(sc[1], key + 32 + 4 * hh, last);
      }
      raise_max(x, sc, c);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        exponentials(x, sc[u], c);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const bf16x8 pf = operand8(sc[u], y);
#pragma unroll
          for (int d = 0; d < 4; ++d)
            x.o[d] = mfma(column8(tv + (32 * u + 16 * y) * kStride + 32 * d), pf, x.o[d]);
        }
      }
    }
    if (more) store(buf ^ 1);
  }

  const float l = both_sum(x.l);
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  const float l2 = log2_sum(x.m, l, c);
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) x.o[d][r] *= inv;
  const int64_t at = ((int64_t)(b * 2 * s.H + 2 * h + map)) * s.N + row;
  if (nsplit > 1) {
    const Parts p = parts_of(A.ws, s, nsplit);
    if (valid) {
      float* o = p.o + (split * p.rows + at) * D + 4 * hh;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(o + 32 * d + 8 * q) =
              make_float4(x.o[d][4 * q], x.o[d][4 * q + 1], x.o[d][4 * q + 2], x.o[d][4 * q + 3]);
      if (hh == 0) p.l[split * p.rows + at] = l2;
    }
    return;
  }
  if (A.lse && valid && hh == 0) A.lse[at] = l2 * kLn2;
  // map 1's rows to map 0's waves through LDS (fp32, rows 528 bytes apart)
  __syncthreads();
  constexpr int kRow = D + 4;
  static_assert(kDiffRows * kRow * 4 <= (int)sizeof(lds), "the second map's rows fit the tiles' LDS");
  float* other = reinterpret_cast<float*>(&lds[0][0]) + (32 * group + l32) * kRow + 4 * hh;
  if (map == 1) {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        *reinterpret_cast<float4*>(other + 32 * d + 8 * q) =
            make_float4(x.o[d][4 * q], x.o[d][4 * q + 1], x.o[d][4 * q + 2], x.o[d][4 * q + 3]);
        if (A.out2 && valid)
          *reinterpret_cast<uint2*>(A.out2 + (((int64_t)b * s.H + h) * s.N + row) * D + 32 * d + 8 * q + 4 * hh) =
              pack4(x.o[d], q);
      }
  }
  __syncthreads();
  if (map == 0 && valid) {
    const float lam = s.lambda[h];
    uint16_t* o = A.out.p + b * A.out.sb + h * A.out.sh + (int64_t)row * A.out.sn + 4 * hh;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float4 y = *reinterpret_cast<const float4*>(other + 32 * d + 8 * q);
        x.o[d][4 * q] = __builtin_fmaf(-lam, y.x, x.o[d][4 * q]);
        x.o[d][4 * q + 1] = __builtin_fmaf(-lam, y.y, x.o[d][4 * q + 1]);
        x.o[d][4 * q + 2] = __builtin_fmaf(-lam, y.z, x.o[d][4 * q + 2]);
        x.o[d][4 * q + 3] = __builtin_fmaf(-lam, y.w, x.o[d][4 * q + 3]);
        *reinterpret_cast<uint2*>(o + 32 * d + 8 * q) = pack4(x.o[d], q);
      }
  }
}

// Few rows over many keys (a token or some drafted ones over a cache): the rows
// of all heads that share a value head -- row r is token r % N of head
// hv per + r / N -- fit one wave's 32.  The keys' bytes bound it, so each wave
// of the workgroup walks every fourth block of 32 keys with both maps on its
// own, through LDS of its own (no barriers), the next block's bytes in flight
// in its registers; the four waves' rows are joined at the end.
template <bool kShared>
__global__ __launch_bounds__(256, 1) void diff_few_kernel(DiffFwd A, int nsplit) {
  constexpr int kBlock = 32, kWaves = 4;
  constexpr int kTileElems = kBlock * kStride;
  constexpr int kKTiles = kShared ? 1 : 2;
  constexpr int kRow = D + 4;
  struct Joined {
    float o[kWaves][2][kFewRows][kRow];
    float m[kWaves][2][kFewRows], l[kWaves][2][kFewRows];
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
  int id = xcd_local_id(blockIdx.x, gridDim.x);
  const int split = id % nsplit;
  id /= nsplit;
  const int hv = id % s.Hv, b = id / s.Hv;
  const int per = s.H / s.Hv, n_rows = per * s.N;
  const Seq sq = sequence(s, b);
  const float c = s.scale * kLog2e;
  const int my = min(l32, n_rows - 1);
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
    const float l = both_sum(x[m].l);
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
      }
    }
  }
  __syncthreads();
  const Parts p = parts_of(A.ws, s, nsplit);
  // one pair of dims of one row a thread and turn
  for (int i = t; i < n_rows * (D / 2); i += 256) {
    const int r = i / (D / 2), d = 2 * (i % (D / 2));
    const int hr = hv * per + r / s.N, n = r % s.N;
    if (n >= sq.qlen) continue;
    float2 o[2];
    float l2[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float top = kNoMax, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds.j.m[w][m][r]);
      o[m] = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f((lds.j.m[w][m][r] - top) * c);
        sum = __builtin_fmaf(f, lds.j.l[w][m][r], sum);
        o[m].x = __builtin_fmaf(f, lds.j.o[w][m][r][d], o[m].x);
        o[m].y = __builtin_fmaf(f, lds.j.o[w][m][r][d + 1], o[m].y);
      }
      const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
      o[m].x *= inv;
      o[m].y *= inv;
      l2[m] = log2_sum(top, sum, c);
    }
    const int64_t at = ((int64_t)(b * 2 * s.H + 2 * hr)) * s.N + n;
    if (nsplit > 1) {
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const int64_t am = split * p.rows + at + m * s.N;
        *reinterpret_cast<float2*>(p.o + am * D + d) = o[m];
        if (d == 0) p.l[am] = l2[m];
      }
    } else {
      const float lam = s.lambda[hr];
      *reinterpret_cast<uint32_t*>(A.out.p + b * A.out.sb + hr * A.out.sh + (int64_t)n * A.out.sn + d) =
          pack_bf16x2(__builtin_fmaf(-lam, o[1].x, o[0].x), __builtin_fmaf(-lam, o[1].y, o[0].y));
      if (A.out2)
        *reinterpret_cast<uint32_t*>(A.out2 + (((int64_t)b * s.H + hr) * s.N + n) * D + d) = pack_bf16x2(o[1].x, o[1].y);
      if (A.lse && d == 0) {
        A.lse[at] = l2[0] * kLn2;
        A.lse[at + s.N] = l2[1] * kLn2;
      }
    }
  }
}

// The splits' results joined: a wave takes a row of an output head, two dims a
// lane, both maps.
__global__ __launch_bounds__(256) void diff_join_kernel(DiffFwd A, int nsplit) {
  const DiffShape& s = A.s;
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= (int64_t)s.B * s.H * s.N) return;
  const int lane = threadIdx.x & 63;
  const int n = (int)(i % s.N);
  const int bh = (int)(i / s.N), h = bh % s.H, b = bh / s.H;
  if (n >= sequence(s, b).qlen) return;
  const Parts p = parts_of(A.ws, s, nsplit);
  float2 o[2];
  float l2[2];
  int64_t at = ((int64_t)(b * 2 * s.H + 2 * h)) * s.N + n;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const int64_t am = at + m * s.N;
    float top = kNoMax, sum = 0.0f;
    for (int u = 0; u < nsplit; ++u) top = fmaxf(top, p.l[u * p.rows + am]);
    o[m] = make_float2(0.0f, 0.0f);
    for (int u = 0; u < nsplit; ++u) {
      const float f = __builtin_amdgcn_exp2f(p.l[u * p.rows + am] - top);
      const float2 x = *reinterpret_cast<const float2*>(p.o + (u * p.rows + am) * D + 2 * lane);
      sum += f;
      o[m].x = __builtin_fmaf(f, x.x, o[m].x);
      o[m].y = __builtin_fmaf(f, x.y, o[m].y);
    }
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    o[m].x *= inv;
    o[m].y *= inv;
    l2[m] = sum > 0.0f ? top + log2f(sum) : -__builtin_inff();
  }
  const float lam = s.lambda[h];
  *reinterpret_cast<uint32_t*>(A.out.p + b * A.out.sb + h * A.out.sh + (int64_t)n * A.out.sn + 2 * lane) =
      pack_bf16x2(__builtin_fmaf(-lam, o[1].x, o[0].x), __builtin_fmaf(-lam, o[1].y, o[0].y));
  if (A.out2) *reinterpret_cast<uint32_t*>(A.out2 + i * D + 2 * lane) = pack_bf16x2(o[1].x, o[1].y);
  if (A.lse && lane < 2) A.lse[at + lane * s.N] = (lane ? l2[1] : l2[0]) * kLn2;
}

// ------------------------------------------------------------------ backward
//
// With X = dout v^T, P_s the maps and delta_s = dout . o_s of a row,
//   dS_0 = P_0 (X - delta_0),  dS_1 = -lambda P_1 (X - delta_1),
//   dq_s = scale dS_s k_s,  dk_s = scale dS_s^T q_s,
//   dv = (P_0 - lambda P_1)^T dout,  dlambda = - sum P_1 X.
// P is found again from the rows' log sums.  Two kernels, one that owns rows
// (dq) and one that owns keys (dk, dv, dlambda): no atomics, and every sum in a
// fixed order.

// Per row and map: the log2 sum that turns scores into P (+inf where the row
// has no keys or is not the sequence's: P is 0 there) and delta.
__global__ __launch_bounds__(256) void diff_stats_kernel(DiffBwd A) {
  const DiffShape& s = A.s;
  const int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (i >= (int64_t)s.B * s.H * s.N) return;
  const int cc = threadIdx.x & 15;
  const int n = (int)(i % s.N);
  const int bh = (int)(i / s.N), h = bh % s.H, b = bh / s.H;
  const bool valid = n < sequence(s, b).qlen;
  float d0 = 0.0f, d1 = 0.0f;
  const int64_t at = ((int64_t)(b * 2 * s.H + 2 * h)) * s.N + n;
  if (valid) {
    float o[8], o1[8], g[8];
    unpack_bf16x8(*reinterpret_cast<const uint4*>(A.out.p + b * A.out.sb + h * A.out.sh + (int64_t)n * A.out.sn + 8 * cc), o);
    unpack_bf16x8(*reinterpret_cast<const uint4*>(A.out2 + i * D + 8 * cc), o1);
    unpack_bf16x8(*reinterpret_cast<const uint4*>(A.dout.p + b * A.dout.sb + h * A.dout.sh + (int64_t)n * A.dout.sn + 8 * cc), g);
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
    const float lse = valid ? A.lse[at + cc * s.N] : 0.0f;
    const bool some = valid && lse > -3e38f;
    A.stats[at + cc * s.N] = make_float2(some ? lse * kLog2e : __builtin_inff(), some ? (cc ? d1 : d0) : 0.0f);
  }
}

// dq of 128 rows of one head, both maps in a wave (X is found once): 32 rows a
// wave over all the keys they see, tiles as in the forward pass.
template <bool kShared>
__global__ __launch_bounds__(256, 1) void diff_dq_kernel(DiffBwd A) {
  constexpr int kTileElems = kDiffKeys * kStride;
  constexpr int kKTiles = kShared ? 1 : 2;
  __shared__ __attribute__((aligned(16))) uint16_t lds[2][(kKTiles + 1) * kTileElems];
  lds_poison(lds, sizeof(lds));
  lds_poison_done();
  const DiffShape& s = A.s;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  const int tiles = (s.N + kDiffRows - 1) / kDiffRows;
  int id = xcd_local_id(blockIdx.x, gridDim.x);
  const int tile = tiles - 1 - id % tiles;
  id /= tiles;
  const int h = id % s.H, b = id / s.H;
  const Seq sq = sequence(s, b);
  const int per = s.H / s.Hv, hv = h / per;
  const int row0 = tile * kDiffRows;
  const int row = row0 + 32 * wave + l32;
  const bool valid = row < sq.qlen;
  const float c = s.scale * kLog2e, lam = s.lambda[h];

  const uint16_t* k0 = A.k.p + b * A.k.sb + (kShared ? hv : 2 * hv) * A.k.sh;
  const uint16_t* k1 = k0 + (kShared ? 0 : A.k.sh);
  const uint16_t* v = A.v.p + b * A.v.sb + hv * A.v.sh;
  bf16x8 qf[2][8], gf[8];
  load_row(qf[0], A.q.p + b * A.q.sb + 2 * h * A.q.sh + (int64_t)row * A.q.sn, valid, hh);
  load_row(qf[1], A.q.p + b * A.q.sb + (2 * h + 1) * A.q.sh + (int64_t)row * A.q.sn, valid, hh);
  load_row(gf, A.dout.p + b * A.dout.sb + h * A.dout.sh + (int64_t)row * A.dout.sn, valid, hh);
  float2 st[2] = {make_float2(__builtin_inff(), 0.0f), make_float2(__builtin_inff(), 0.0f)};
  if (valid) {
    const int64_t at = ((int64_t)(b * 2 * s.H + 2 * h)) * s.N + row;
    st[0] = A.stats[at];
    st[1] = A.stats[at + s.N];
  }

  const int last = min(row + sq.shift, sq.klen - 1);
  const int last_row = min(row0 + kDiffRows, sq.qlen) - 1;
  const int kend = row0 < sq.qlen ? min(last_row + sq.shift, sq.klen - 1) + 1 : 0;
  const int wave_row = row0 + 32 * wave;
  const int all_to = min(wave_row + sq.shift, sq.klen - 1);
  const int none_from = wave_row < sq.qlen ? min(wave_row + 31 + sq.shift, sq.klen - 1) : -1;

  f32x16 dq[2][4] = {};
  const int tr = column_offset(lane);
  Stage<kDiffKeys, 256> sk0, sk1, sv;
  auto load = [&](int key) __attribute__((always_inline)) {
    sk0.load(k0, A.k.sn, key, kend, t);
    if (!kShared) sk1.load(k1, A.k.sn, key, kend, t);
    sv.load(v, A.v.sn, key, kend, t);
  };
  auto store = [&](int buf) __attribute__((always_inline)) {
    sk0.store(lds[buf], t);
    if (!kShared) sk1.store(lds[buf] + kTileElems, t);
    sv.store(lds[buf] + kKTiles * kTileElems, t);
  };
  if (kend > 0) {
    load(0);
    store(0);
  }
  int buf = 0;
  for (int key = 0; key < kend; key += kDiffKeys, buf ^= 1) {
    __syncthreads();
    const bool more = key + kDiffKeys < kend;
    if (more) load(key + kDiffKeys);
    if (key <= none_from) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint16_t* tk0 = lds[buf] + 32 * u * kStride;
        const uint16_t* tk1 = kShared ? tk0 : tk0 + kTileElems;
        const uint16_t* tv = lds[buf] + kKTiles * kTileElems + 32 * u * kStride;
        f32x16 s0 = scores(tk0, qf[0], lane), s1 = scores(tk1, qf[1], lane), x = scores(tv, gf, lane);
        if (key + 32 * u + 31 > all_to) {
          mask(s0, key + 32 * u + 4 * hh, last);
          mask(s1, key + 32 * u + 4 * hh, last);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s0[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s0[r], c, -st[0].x)) * (x[r] - st[0].y);
          s1[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s1[r], c, -st[1].x)) * (x[r] - st[1].y);
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const bf16x8 d0 = operand8(s0, y), d1 = operand8(s1, y);
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const bf16x8 kf = column8(tk0 + 16 * y * kStride + 32 * d + tr);
            dq[0][d] = mfma(kf, d0, dq[0][d]);
            dq[1][d] = mfma(kShared ? kf : column8(tk1 + 16 * y * kStride + 32 * d + tr), d1, dq[1][d]);
          }
        }
      }
    }
    if (more) store(buf ^ 1);
  }
  if (row < s.N) {  // zero behind the sequence
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const float f = m ? -lam * s.scale : s.scale;
      uint16_t* o = A.dq.p + b * A.dq.sb + (2 * h + m) * A.dq.sh + (int64_t)row * A.dq.sn + 4 * hh;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
#pragma unroll
        for (int r = 0; r < 16; ++r) dq[m][d][r] = valid ? dq[m][d][r] * f : 0.0f;
#pragma unroll
        for (int q = 0; q < 4; ++q) *reinterpret_cast<uint2*>(o + 32 * d + 8 * q) = pack4(dq[m][d], q);
      }
    }
  }
}

// dk, dv of 128 keys of one value head, 32 keys a wave, over the rows of every
// head of its group (so a shared head's gradient is summed in registers, heads
// in order); dlambda's parts of these keys.
constexpr int kBwdRows = 32;  // query rows of a tile
template <bool kShared>
__global__ __launch_bounds__(256, 1) void diff_dkv_kernel(DiffBwd A) {
  constexpr int kTileElems = kBwdRows * kStride;
  constexpr int kK = kShared ? 1 : 2;
  __shared__ __attribute__((aligned(16))) uint16_t lds[2][3 * kTileElems];
  __shared__ __attribute__((aligned(16))) float rowstat[2][4][kBwdRows];  // log2 sums of the maps, deltas of the maps
  lds_poison(lds, sizeof(lds));
  lds_poison(rowstat, sizeof(rowstat));
  lds_poison_done();
  const DiffShape& s = A.s;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63, hh = lane >> 5, l32 = lane & 31;
  const int tiles = (s.M + kDiffRows - 1) / kDiffRows;
  int id = xcd_local_id(blockIdx.x, gridDim.x);
  const int tile = id % tiles;  // causal: the long columns first
  id /= tiles;
  const int hv = id % s.Hv, b = id / s.Hv;
  const Seq sq = sequence(s, b);
  const int per = s.H / s.Hv;
  const int key0 = tile * kDiffRows;
  const int key = key0 + 32 * wave + l32;
  const bool valid = key < sq.klen;
  const float c = s.scale * kLog2e;

  bf16x8 kf[kK][8], vf[8];
  const uint16_t* kp = A.k.p + b * A.k.sb + (kShared ? hv : 2 * hv) * A.k.sh + (int64_t)key * A.k.sn;
  load_row(kf[0], kp, valid, hh);
  if (!kShared) load_row(kf[kK - 1], kp + A.k.sh, valid, hh);
  load_row(vf, A.v.p + b * A.v.sb + hv * A.v.sh + (int64_t)key * A.v.sn, valid, hh);

  // rows that see any key of this tile: from key0 - shift on
  const int first = key0 < sq.klen ? min(max(key0 - sq.shift, 0), sq.qlen) / kBwdRows * kBwdRows : sq.qlen;
  const int wave_last_key = key0 + 32 * wave + 31;

  f32x16 dv[4] = {}, dk[kK][4] = {};
  const int tr = column_offset(lane);
  for (int u = 0; u < per; ++u) {
    const int h = hv * per + u;
    const float lam = s.lambda[h];
    const uint16_t* q0 = A.q.p + b * A.q.sb + 2 * h * A.q.sh;
    const uint16_t* q1 = q0 + A.q.sh;
    const uint16_t* g = A.dout.p + b * A.dout.sb + h * A.dout.sh;
    const float2* st = A.stats + ((int64_t)(b * 2 * s.H + 2 * h)) * s.N;
    float dlam = 0.0f;
    Stage<kBwdRows, 256> s0, s1, sg;
    float2 stat;
    auto load = [&](int row) __attribute__((always_inline)) {
      s0.load(q0, A.q.sn, row, sq.qlen, t);
      s1.load(q1, A.q.sn, row, sq.qlen, t);
      sg.load(g, A.dout.sn, row, sq.qlen, t);
      const int r = row + (t & 31);
      stat = make_float2(__builtin_inff(), 0.0f);
      if (t < 64 && r < sq.qlen) stat = st[(t >> 5) * s.N + r];
    };
    auto store = [&](int buf) __attribute__((always_inline)) {
      s0.store(lds[buf], t);
      s1.store(lds[buf] + kTileElems, t);
      sg.store(lds[buf] + 2 * kTileElems, t);
      if (t < 64) {
        rowstat[buf][t >> 5][t & 31] = stat.x;
        rowstat[buf][2 + (t >> 5)][t & 31] = stat.y;
      }
    };
    __syncthreads();  // the last head's tiles are read
    if (first < sq.qlen) {
      load(first);
      store(0);
    }
    int buf = 0;
    for (int row = first; row < sq.qlen; row += kBwdRows, buf ^= 1) {
      __syncthreads();
      const bool more = row + kBwdRows < sq.qlen;
      if (more) load(row + kBwdRows);
      if (row + kBwdRows - 1 + sq.shift >= key0 + 32 * wave) {
        const uint16_t *t0 = lds[buf], *t1 = t0 + kTileElems, *tg = t1 + kTileElems;
        // rows of q (lane) times keys: result row = row of q, column = key
        f32x16 p0 = {}, p1 = {}, x = {};
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
          p0 = mfma(row8(t0, lane, kk), kf[0][kk], p0);
          p1 = mfma(row8(t1, lane, kk), kf[kK - 1][kk], p1);
          x = mfma(row8(tg, lane, kk), vf[kk], x);
        }
        const bool edge = wave_last_key >= sq.klen || wave_last_key > row + sq.shift;
        float l0[16], l1[16], e0[16], e1[16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          *reinterpret_cast<float4*>(&l0[4 * q]) = *reinterpret_cast<const float4*>(&rowstat[buf][0][8 * q + 4 * hh]);
          *reinterpret_cast<float4*>(&l1[4 * q]) = *reinterpret_cast<const float4*>(&rowstat[buf][1][8 * q + 4 * hh]);
          *reinterpret_cast<float4*>(&e0[4 * q]) = *reinterpret_cast<const float4*>(&rowstat[buf][2][8 * q + 4 * hh]);
          *reinterpret_cast<float4*>(&e1[4 * q]) = *reinterpret_cast<const float4*>(&rowstat[buf][3][8 * q + 4 * hh]);
        }
        f32x16 mix;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float a = __builtin_amdgcn_exp2f(__builtin_fmaf(p0[r], c, -l0[r]));
          float d = __builtin_amdgcn_exp2f(__builtin_fmaf(p1[r], c, -l1[r]));
          if (edge) {
            const bool seen = valid && key <= row + 8 * (r >> 2) + 4 * hh + (r & 3) + sq.shift;
            a = seen ? a : 0.0f;
            d = seen ? d : 0.0f;
          }
          dlam = __builtin_fmaf(d, x[r], dlam);
          mix[r] = __builtin_fmaf(-lam, d, a);
          p0[r] = a * (x[r] - e0[r]);
          p1[r] = -lam * d * (x[r] - e1[r]);
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const bf16x8 fm = operand8(mix, y), f0 = operand8(p0, y), f1 = operand8(p1, y);
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const int at = 16 * y * kStride + 32 * d + tr;
            dv[d] = mfma(column8(tg + at), fm, dv[d]);
            dk[0][d] = mfma(column8(t0 + at), f0, dk[0][d]);
            dk[kK - 1][d] = mfma(column8(t1 + at), f1, dk[kK - 1][d]);
          }
        }
      }
      if (more) store(buf ^ 1);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) dlam += __shfl_xor(dlam, m);
    if (lane == 0) A.partial[((int64_t)h * s.B + b) * A.parts + tile * 4 + wave] = dlam;
  }
  if (key < s.M) {  // zero behind the sequence
    uint16_t* o = A.dv.p + b * A.dv.sb + hv * A.dv.sh + (int64_t)key * A.dv.sn + 4 * hh;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
#pragma unroll
      for (int r = 0; r < 16; ++r) dv[d][r] = valid ? dv[d][r] : 0.0f;
#pragma unroll
      for (int q = 0; q < 4; ++q) *reinterpret_cast<uint2*>(o + 32 * d + 8 * q) = pack4(dv[d], q);
    }
#pragma unroll
    for (int m = 0; m < kK; ++m) {
      uint16_t* ok = A.dk.p + b * A.dk.sb + ((kShared ? hv : 2 * hv) + m) * A.dk.sh + (int64_t)key * A.dk.sn + 4 * hh;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[m][d][r] = valid ? dk[m][d][r] * s.scale : 0.0f;
#pragma unroll
        for (int q = 0; q < 4; ++q) *reinterpret_cast<uint2*>(ok + 32 * d + 8 * q) = pack4(dk[m][d], q);
      }
    }
  }
}

// dlambda of a head: its parts summed in one order, in 64 bits.
__global__ __launch_bounds__(256) void diff_dlambda_kernel(DiffBwd A) {
  __shared__ double sum[256];
  const float* p = A.partial + (int64_t)blockIdx.x * A.s.B * A.parts;
  double x = 0.0;
  for (int64_t i = threadIdx.x; i < (int64_t)A.s.B * A.parts; i += 256) x += (double)p[i];
  sum[threadIdx.x] = x;
  __syncthreads();
  for (int n = 128; n > 0; n >>= 1) {
    if ((int)threadIdx.x < n) sum[threadIdx.x] += sum[threadIdx.x + n];
    __syncthreads();
  }
  if (threadIdx.x == 0) A.dlambda[blockIdx.x] = (float)-sum[0];
}

}  // namespace

DiffPlan diff_plan(const DiffShape& s) {
  DiffPlan p;
  p.few = (int64_t)(s.H / s.Hv) * s.N <= kFewRows;
  const int64_t wgs = p.few ? (int64_t)s.B * s.Hv : (int64_t)s.B * s.H * ((s.N + kDiffRows - 1) / kDiffRows);
  // the chip's 256 CUs hold one workgroup each; a split has 512 keys or more
  int64_t n = 256 / wgs;
  const int64_t most = s.M / 512;
  if (n > most) n = most;
  p.nsplit = (int)(n < 1 ? 1 : n);
  return p;
}

size_t diff_fwd_bytes(const DiffShape& s) {
  const DiffPlan p = diff_plan(s);
  return p.nsplit > 1 ? (size_t)p.nsplit * s.B * 2 * s.H * s.N * (D + 1) * sizeof(float) : 0;
}

hipError_t launch_diff_fwd(const DiffFwd& a, hipStream_t stream) {
  const DiffShape& s = a.s;
  const DiffPlan p = diff_plan(s);
  const bool shared = s.Hk == s.Hv;
  if (p.few) {
    const dim3 grid((unsigned)((int64_t)s.B * s.Hv * p.nsplit));
    if (shared)
      hipLaunchKernelGGL(diff_few_kernel<true>, grid, dim3(256), 0, stream, a, p.nsplit);
    else
      hipLaunchKernelGGL(diff_few_kernel<false>, grid, dim3(256), 0, stream, a, p.nsplit);
  } else {
    const dim3 grid((unsigned)((int64_t)s.B * s.H * ((s.N + kDiffRows - 1) / kDiffRows) * p.nsplit));
    if (shared)
      hipLaunchKernelGGL(diff_fwd_kernel<true>, grid, dim3(512), 0, stream, a, p.nsplit);
    else
      hipLaunchKernelGGL(diff_fwd_kernel<false>, grid, dim3(512), 0, stream, a, p.nsplit);
  }
  if (p.nsplit > 1) {
    const int64_t rows = (int64_t)s.B * s.H * s.N;
    hipLaunchKernelGGL(diff_join_kernel, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, a, p.nsplit);
  }
  return hipGetLastError();
}

size_t diff_bwd_bytes(const DiffShape& s, size_t* partial_at, int* parts) {
  const size_t stats = ((size_t)s.B * 2 * s.H * s.N * sizeof(float2) + 255) & ~(size_t)255;
  *partial_at = stats;
  *parts = 4 * ((s.M + kDiffRows - 1) / kDiffRows);
  return stats + (size_t)s.H * s.B * *parts * sizeof(float);
}

hipError_t launch_diff_bwd(const DiffBwd& a, hipStream_t stream) {
  const DiffShape& s = a.s;
  const int64_t rows = (int64_t)s.B * s.H * s.N;
  const bool shared = s.Hk == s.Hv;
  hipLaunchKernelGGL(diff_stats_kernel, dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, stream, a);
  const dim3 gq((unsigned)((int64_t)s.B * s.H * ((s.N + kDiffRows - 1) / kDiffRows)));
  const dim3 gk((unsigned)((int64_t)s.B * s.Hv * ((s.M + kDiffRows - 1) / kDiffRows)));
  if (shared) {
    hipLaunchKernelGGL(diff_dq_kernel<true>, gq, dim3(256), 0, stream, a);
    hipLaunchKernelGGL(diff_dkv_kernel<true>, gk, dim3(256), 0, stream, a);
  } else {
    hipLaunchKernelGGL(diff_dq_kernel<false>, gq, dim3(256), 0, stream, a);
    hipLaunchKernelGGL(diff_dkv_kernel<false>, gk, dim3(256), 0, stream, a);
  }
  hipLaunchKernelGGL(diff_dlambda_kernel, dim3((unsigned)s.H), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sol
