// Linear attention with a decay for each head (sol_lin_attn_fwd, _bwd, _step).
//
//   S_t = e^g S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t      (S: 128 x 128, fp32)
//
// Over a chunk of C tokens with the state S before it this is
//   o_i = scale [ sum_{j<=i} e^{g(i-j)} (q_i.k_j) v_j  +  e^{g(i+1)} q_i^T S ]
//   S'  = e^{gC} S + sum_j e^{g(C-1-j)} k_j v_j^T
// three matrix products a chunk beside the C x C one, all on MFMA.
//
// The gradients are the same scan with other operands.  With dS_T the gradient
// of the final state,
//   dq_i = scale [ sum_{j<=i} e^{g(i-j)} (do_i.v_j) k_j + e^{g(i+1)} S_0 do_i .. ]
// is the scan of (do, v, k) on the transposed state, and, tokens walked from
// the last to the first,
//   dk = scan of (v, do, q),  dv = scan of (k, q, do),
//   dS_{t-1} = e^g (dS_t + scale q_t do_t^T)
// with the state dS.  One kernel serves all four: it computes
//   y_i = sum_{j<=i} p e^{g(i-j)} (a_i.b_j) c_j + r e^{g(i+off)} a_i^T S
//   S'  = e^{gC} S + sum_j u e^{g(C-off-j)} b_j c_j^T
// off = 1 forwards and 0 backwards (where a token's own row meets the state
// before it is decayed), tokens reversed by a negative row stride.
#include <hip/hip_runtime.h>

#include "sol_ops.h"
#include "sol_tiles.h"

namespace sol {
namespace {

constexpr int kThreads = 256;
constexpr int kC = kLinRows;
constexpr int kTile = 2 * kTile32;  // bytes of a chunk's rows

// One scan.  A launch takes up to kMaxScans of the same shape (the backward
// pass's), whose workgroups take turns.
constexpr int kMaxScans = 3;
struct Scan {
  Rows a, b, c;
  int a_div, b_div, c_div;  // head h of the scan reads head h / div
  void* y;                  // bf16, or fp32 when y_f32
  int64_t y_b, y_h, y_n;
  int y_f32;
  const float* state_in;  // the state before the first token
  int state_t;            // state_in is held transposed
  float* state_out;       // the state after the last token (may be null)
  float* before;          // several segments: the states before them, [slab][segment][128][128]
  float p, r, u;
  int off;
  int reverse;    // walk the tokens from the last one
  int zero_tail;  // write zeros to the rows behind the sequence
};
// The states that segments add, found in one pass for the scans that need them.
struct SegmentStates {
  Rows b, c;
  int b_div, c_div;
  const float* state_in;
  int state_t;
  float* state_out;
  float* local;       // in: what the segments add; out: the states before them
  float* transposed;  // the same, transposed (may be null)
  float u;
  int off;
  int reverse;
};
struct Shape {
  const float* log_decay;
  const int32_t* lens;
  int H, N, seg_rows, nseg;
};
struct ScanArgs {
  Shape sh;
  Scan scan[kMaxScans];
  int n;
};
struct StateArgs {
  Shape sh;
  SegmentStates st[2];
  int n;
};

__device__ __forceinline__ float decay_log2(const float* log_decay, int h) {
  // -inf (a head without memory) becomes a number whose multiple by 0 is 0
  return fmaxf(log_decay[h], -1e30f) * 1.44269504088896341f;
}
__device__ __forceinline__ int length_of(const Shape& s, int b) {
  return s.lens ? __builtin_amdgcn_readfirstlane(min(max(s.lens[b], 0), s.N)) : s.N;
}

// The wave's 32 columns of the state as four 32 x 32 MFMA results.  Its rows are
// dealt to the results so that a lane's eight consecutive registers are eight
// consecutive rows -- the operand of a product with eight consecutive dims of a
// row of a: register r of result t is row state_row, column 32 wave + l % 32.
struct State {
  f32x16 s[4];
};
__device__ __forceinline__ int state_row(int t, int r, int hh) {
  return 32 * t + 16 * (r >> 3) + 8 * hh + (r & 7);
}
__device__ __forceinline__ void load_state(State& st, const float* p, bool transposed, int col, int hh) {
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = state_row(t, r, hh);
      st.s[t][r] = transposed ? p[col * D + row] : p[row * D + col];
    }
}
__device__ __forceinline__ void store_state(const State& st, float* p, int col, int hh) {
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) p[state_row(t, r, hh) * D + col] = st.s[t][r];
}
// This lane's place in the transpose reads of b: column l % 32 with bits 2 and 3
// exchanged, which deals the rows of the state as above.
__device__ __forceinline__ int state_col_place(int lane) {
  const int g16 = lane >> 4, i16 = lane & 15, r = 4 * (g16 >> 1) + (i16 >> 2);
  const int x = (i16 & 1) * 2 + ((i16 >> 1) & 1);  // four columns from 4 x
  return r * 128 + ((2 * (g16 & 1) + (x >> 1)) ^ swizzle(r)) * 16 + (x & 1) * 8;
}

// S = (1 - fade) S + b^T (c w): the decay is taken off as a difference, so that
// its rounding is relative to what is lost and slow heads (e^{64 g} next to 1)
// do not drift over long sequences.  A weighted row of c enters rounded to bf16,
// and with kExact (a state that is a result of its own) as the sum of two bf16,
// the rounding and the rounding of the rest, 2^-17 together.
template <bool kExact>
__device__ __forceinline__ void update_state(State& st, float fade, const uint8_t* tb, const bf16x8 (&cf)[4],
                                             const float* w, int place, int hh) {
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.s[t][r] = __builtin_fmaf(st.s[t][r], -fade, st.s[t][r]);
  bf16x8 hi[4], lo[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    const float4 w0 = *reinterpret_cast<const float4*>(w + 16 * ks + 4 * hh);
    const float4 w1 = *reinterpret_cast<const float4*>(w + 16 * ks + 8 + 4 * hh);
    float x[8], rest[8];
    unpack_bf16x8(__builtin_bit_cast(uint4, cf[ks]), x);
    x[0] *= w0.x; x[1] *= w0.y; x[2] *= w0.z; x[3] *= w0.w;
    x[4] *= w1.x; x[5] *= w1.y; x[6] *= w1.z; x[7] *= w1.w;
    const uint4 h = pack_bf16x8(x);
    hi[ks] = __builtin_bit_cast(bf16x8, h);
    if (kExact) {
      unpack_bf16x8(h, rest);
#pragma unroll
      for (int i = 0; i < 8; ++i) rest[i] = x[i] - rest[i];
      lo[ks] = __builtin_bit_cast(bf16x8, pack_bf16x8(rest));
    }
  }
  // fragments four reads ahead
  bf16x8 ring[4];
#pragma unroll
  for (int f = 0; f < 4; ++f) ring[f] = col_frag(tb + place, 0, f);
  slot_end();
  // (the decayed state and the weighted rows two wait states before an MFMA reads them)
  asm volatile("s_nop 1" : "+v"(st.s[0]), "+v"(st.s[1]), "+v"(st.s[2]), "+v"(st.s[3]));
#pragma unroll
  for (int f = 0; f < 16; ++f) {
    const int ks = f >> 2, t = f & 3;
    score(st.s[t], ring[f & 3], hi[ks]);
    if (kExact) score(st.s[t], ring[f & 3], lo[ks]);
    if (f + 4 < 16) ring[f & 3] = col_frag(tb + place, (f + 4) >> 2, t);
    slot_end();
  }
}

// A value that all lanes hold, in a scalar register (a division leaves it in a
// vector one).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The walk of a workgroup over its segment's chunks: rows [row0, rows) of the
// sequence in walking order.
struct Walk {
  int b, h, seg, len, row0, rows, chunks;
  float g2;
};
__device__ __forceinline__ Walk make_walk(const Shape& s, int id) {
  Walk w;
  const int slab = uniform(id / s.nseg);
  w.seg = id - slab * s.nseg;
  w.b = uniform(slab / s.H);
  w.h = slab - w.b * s.H;
  w.len = length_of(s, w.b);
  w.row0 = w.seg * s.seg_rows;
  w.rows = min(w.row0 + s.seg_rows, w.len);
  w.chunks = w.rows > w.row0 ? (w.rows - w.row0 + kC - 1) / kC : 0;
  w.g2 = decay_log2(s.log_decay, w.h);
  return w;
}
__device__ __forceinline__ const uint16_t* slab_of(const Rows& r, const Walk& w, int div) {
  return r.p + w.b * r.sb + (w.h / div) * r.sh;
}
// A chunk's 64 rows of one tensor into LDS, four kilobytes a wave.  Rows past
// the sequence are its last ones again (their weights are 0, and no result of
// theirs is stored).
__device__ __forceinline__ void copy_chunk(uint32_t lds, const uint16_t* slab, int64_t sn, const Walk& w, int chunk,
                                           int reverse, int wave, int lane) {
  const int i = w.row0 + chunk * kC, m = min(kC, w.rows - i);
  const uint64_t at = reinterpret_cast<uint64_t>(slab + (int64_t)(reverse ? w.len - i - m : i) * sn);
  // (a vector instruction's scalar result is five wait states from a copy's address)
  const uint32_t lo = uniform((int)(uint32_t)at), hi = uniform((int)(uint32_t)(at >> 32));
  const void* base = reinterpret_cast<const void*>(lo | (uint64_t)hi << 32);
  asm volatile("s_nop 4" : "+s"(base));
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int r = min(8 * (2 * wave + u) + (lane >> 3), m - 1);
    const uint32_t off = copy_offset(reverse ? m - 1 - r : r, sn, lane);
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (2 * wave + u) * kRowBlock);
    copy_1k(to, base, off);
    copy_1k(to + 1024, base, off + 128);
  }
}
constexpr int kChunkCopies = 4;  // of one tensor, by each wave

// w[j] = u e^{g(m - off - j)} for the m rows of a chunk, 0 past them.
__device__ __forceinline__ void fill_weights(float* w, float u, int off, float g2, int m) {
  const int j = threadIdx.x;
  if (j < kC) w[j] = j < m ? u * __builtin_amdgcn_exp2f(g2 * (float)max(m - off - j, 0)) : 0.0f;
}
__device__ __forceinline__ float fade_of(float g2, int m) { return -expm1f(g2 * 0.693147180559945309f * (float)m); }

// The states that segments add, from zero: one pass over b and c.
constexpr int kStateRing = 4;
template <bool kExact>
__global__ __launch_bounds__(kThreads, 2) void lin_state_kernel(StateArgs A) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kStateRing][2][kTile];
  __shared__ __attribute__((aligned(16))) float wt[2][kC];
  lds_poison(lds, sizeof(lds));
  lds_poison(wt, sizeof(wt));
  lds_poison_done();
  const int all = xcd_local_id(blockIdx.x, gridDim.x);
  const int id = uniform(all / A.n);
  const SegmentStates S = A.st[all - id * A.n];
  const Walk W = make_walk(A.sh, id);
  // the last segment's state is wanted by the final state alone
  if (W.seg == A.sh.nseg - 1 && !S.state_out) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hh = lane >> 5, l32 = lane & 31;
  const int place = state_col_place(lane), c_place = col_place(lane);
  const uint16_t *pb = slab_of(S.b, W, S.b_div), *pc = slab_of(S.c, W, S.c_div);
  const uint32_t at0 = lds_address(&lds[0][0][0]);
  auto copy = [&](int i) __attribute__((always_inline)) {
    const int chunk = min(i, W.chunks - 1);  // (past the last one: again, not used)
    const uint32_t to = at0 + (i % kStateRing) * (2 * kTile);
    copy_chunk(to, pb, S.b.sn, W, chunk, S.reverse, wave, lane);
    copy_chunk(to + kTile, pc, S.c.sn, W, chunk, S.reverse, wave, lane);
  };
  State st{};
  if (W.chunks > 0) {
    float fade = fade_of(W.g2, kC);
    fill_weights(wt[0], S.u, S.off, W.g2, min(kC, W.rows - W.row0));
    all_landed();
    copy(0);
    copy(1);
    for (int i = 0; i < W.chunks; ++i) {
      const int m = min(kC, W.rows - W.row0 - i * kC);
      if (m < kC) {  // the last chunk's own (the other buffer: this one may be in use)
        if (i > 0) fill_weights(wt[1], S.u, S.off, W.g2, m);
        fade = fade_of(W.g2, m);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      copies_landed<2 * kChunkCopies>();
      copy(i + 2);
      const uint8_t* tb = lds[i % kStateRing][0];
      bf16x8 cf[4];
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) cf[ks] = col_frag(lds[i % kStateRing][1] + c_place, ks, wave);
      update_state<kExact>(st, fade, tb, cf, wt[m < kC && i > 0], place, hh);
    }
    copies_landed<0>();
  }
  settle(st.s[0], st.s[1]);
  settle(st.s[2], st.s[3]);
  store_state(st, S.local + (int64_t)id * kStateElems, 32 * wave + l32, hh);
}

// The states before each segment, from what the segments add: in place, one
// workgroup per slab and 1,024 of its state's values, eight segments' loads in
// flight.
__global__ __launch_bounds__(kThreads) void lin_join_kernel(StateArgs A) {
  const SegmentStates& S = A.st[blockIdx.x % A.n];
  const int slab = blockIdx.x / A.n >> 4, part = (blockIdx.x / A.n) & 15;
  const int b = slab / A.sh.H, h = slab - b * A.sh.H;
  const int len = length_of(A.sh, b), nseg = A.sh.nseg;
  const float g2 = decay_log2(A.sh.log_decay, h);
  const int e = part * 1024 + threadIdx.x * 4, row = e >> 7, col = e & 127;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (S.state_in) {
    const float* p = S.state_in + (int64_t)slab * kStateElems;
    s = S.state_t ? make_float4(p[col * D + row], p[(col + 1) * D + row], p[(col + 2) * D + row], p[(col + 3) * D + row])
                  : *reinterpret_cast<const float4*>(p + e);
  }
  float* seg = S.local + (int64_t)slab * nseg * kStateElems;
  float* tr = S.transposed ? S.transposed + (int64_t)slab * nseg * kStateElems + col * D + row : nullptr;
  const float whole = fade_of(g2, A.sh.seg_rows);
  const int last = S.state_out ? nseg : nseg - 1;  // segments whose own state was found
  constexpr int kBatch = 8;
  for (int i0 = 0; i0 < nseg; i0 += kBatch) {
    float4 x[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i0 + u < last) x[u] = *reinterpret_cast<const float4*>(seg + (int64_t)(i0 + u) * kStateElems + e);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int i = i0 + u;
      if (i < nseg) {
        *reinterpret_cast<float4*>(seg + (int64_t)i * kStateElems + e) = s;
        if (tr) {
          float* t = tr + (int64_t)i * kStateElems;
          t[0] = s.x;
          t[D] = s.y;
          t[2 * D] = s.z;
          t[3 * D] = s.w;
        }
        const int m = min(max(len - i * A.sh.seg_rows, 0), A.sh.seg_rows);
        const float fade = m == A.sh.seg_rows ? whole : fade_of(g2, m);
        s.x = __builtin_fmaf(s.x, -fade, s.x) + x[u].x;
        s.y = __builtin_fmaf(s.y, -fade, s.y) + x[u].y;
        s.z = __builtin_fmaf(s.z, -fade, s.z) + x[u].z;
        s.w = __builtin_fmaf(s.w, -fade, s.w) + x[u].w;
      }
    }
  }
  if (S.state_out) *reinterpret_cast<float4*>(S.state_out + (int64_t)slab * kStateElems + e) = s;
}

// a b^T of 32 rows each over the 128 dims, in two halves (two chains of MFMAs).
__device__ __forceinline__ void tile_product(f32x16 (&s)[2], const bf16x8 (&bf)[8], const bf16x8 (&af)[8]) {
  score_first(s[0], bf[0], af[0]);
  score_first(s[1], bf[1], af[1]);
#pragma unroll
  for (int kk = 2; kk < 8; ++kk) score(s[kk & 1], bf[kk], af[kk]);
}

// y over a segment.  A wave owns 32 columns of the state and of y: the state
// stays in its registers (64 a lane), where an MFMA leaves it and the next one
// takes it as an operand (rounded to bf16 there, as y is a bf16 result: both
// roundings are of the same size).  The C x C products are shared: waves 0 to 2
// find the three 32 x 32 tiles on and below the diagonal, and pass them round
// in the order the next product reads them.
//
// Its bytes bound it: a CU's share of a copy's rate is 64 KB (a chunk's a, b, c
// and y) in 6,800 cycles, the products of a chunk take 1,500 of the matrix
// cores.  So one workgroup a CU, the chunks straight into LDS in a ring of
// three, two on their way.
constexpr int kScanRing = 3;
template <bool kExact>
__global__ __launch_bounds__(kThreads, 2) void lin_scan_kernel(ScanArgs A) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kScanRing][3][kTile];
  __shared__ __attribute__((aligned(16))) uint4 pf[3][2][64];  // tiles (0,0), (1,0), (1,1): 16 columns, lane
  __shared__ __attribute__((aligned(16))) float wt[2][kC];
  lds_poison(lds, sizeof(lds));
  lds_poison(pf, sizeof(pf));
  lds_poison(wt, sizeof(wt));
  lds_poison_done();
  const int all = xcd_local_id(blockIdx.x, gridDim.x);
  const int id = uniform(all / A.n);
  const Scan S = A.scan[all - id * A.n];
  const Walk W = make_walk(A.sh, id);
  const int slab = W.b * A.sh.H + W.h;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hh = lane >> 5, l32 = lane & 31;
  const int col = 32 * wave + l32;
  const int64_t y0 = W.b * S.y_b + W.h * S.y_h;

  if (S.zero_tail) {  // rows of this segment behind the sequence
    const int r = threadIdx.x >> 4, cc = threadIdx.x & 15;
    const int end = min(W.row0 + A.sh.seg_rows, A.sh.N);
    for (int i = max(W.row0, W.len) + r; i < end; i += 16) {
      const int64_t at = y0 + (int64_t)i * S.y_n + cc * 8;
      if (S.y_f32) {
        float4* y = reinterpret_cast<float4*>(static_cast<float*>(S.y) + at);
        y[0] = y[1] = make_float4(0.f, 0.f, 0.f, 0.f);
      } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(S.y) + at) = make_uint4(0, 0, 0, 0);
      }
    }
  }
  if (W.chunks == 0) {  // (of a sequence without tokens, the first and last segment)
    if (A.sh.nseg == 1 && S.state_out)
      for (int e = threadIdx.x; e < kStateElems; e += kThreads)
        S.state_out[(int64_t)slab * kStateElems + e] =
            !S.state_in ? 0.0f : S.state_in[(int64_t)slab * kStateElems + (S.state_t ? (e & 127) * D + (e >> 7) : e)];
    return;
  }

  const RowPlace rp = row_place(lane);
  const int place = state_col_place(lane), c_place = col_place(lane);
  const uint16_t *pa = slab_of(S.a, W, S.a_div), *pb = slab_of(S.b, W, S.b_div), *pc = slab_of(S.c, W, S.c_div);
  const uint32_t at0 = lds_address(&lds[0][0][0]);
  auto copy = [&](int i) __attribute__((always_inline)) {
    const int chunk = min(i, W.chunks - 1);  // (past the last one: again, not used)
    const uint32_t to = at0 + (i % kScanRing) * (3 * kTile);
    copy_chunk(to, pa, S.a.sn, W, chunk, S.reverse, wave, lane);
    copy_chunk(to + kTile, pb, S.b.sn, W, chunk, S.reverse, wave, lane);
    copy_chunk(to + 2 * kTile, pc, S.c.sn, W, chunk, S.reverse, wave, lane);
  };
  State st{};
  if (A.sh.nseg > 1)
    load_state(st, S.before + (int64_t)id * kStateElems, false, col, hh);
  else if (S.state_in)
    load_state(st, S.state_in + (int64_t)slab * kStateElems, S.state_t, col, hh);

  // this wave's tile of the C x C product: rows 32 I + .. of a, 32 J + .. of b,
  // held transposed (lane: row of a), and its weights
  const int I = wave == 0 ? 0 : 1, J = wave == 2 ? 1 : 0;
  float dec[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int gap = (32 * I + l32) - (32 * J + 8 * (r >> 2) + 4 * hh + (r & 3));
    dec[r] = gap >= 0 ? S.p * __builtin_amdgcn_exp2f(W.g2 * (float)gap) : 0.0f;
  }
  const float win[2] = {S.r * __builtin_amdgcn_exp2f(W.g2 * (float)(l32 + S.off)),
                        S.r * __builtin_amdgcn_exp2f(W.g2 * (float)(32 + l32 + S.off))};
  float fade = fade_of(W.g2, kC);
  fill_weights(wt[0], S.u, S.off, W.g2, min(kC, W.rows - W.row0));
  constexpr int kStores = 8;  // of y, by each wave and chunk
  all_landed();
  copy(0);
  copy(1);
  for (int i = 0; i < W.chunks; ++i) {
    const int row = W.row0 + i * kC, m = min(kC, W.rows - row);
    if (m < kC) {  // the last chunk's own (the other buffer: this one may be in use)
      if (i > 0) fill_weights(wt[1], S.u, S.off, W.g2, m);
      fade = fade_of(W.g2, m);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    // this chunk's copies: behind them the next one's, and from the second
    // chunk on the last one's stores (every chunk but the last stores 8 times)
    if (i == 0)
      copies_landed<3 * kChunkCopies>();
    else
      copies_landed<3 * kChunkCopies + kStores>();
    copy(i + 2);
    const uint8_t *ta = lds[i % kScanRing][0], *tb = lds[i % kScanRing][1], *tc = lds[i % kScanRing][2];
    bf16x8 af[2][8], cf[4];
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) af[0][kk] = row_frag(ta, rp, kk);
    if (wave < 3) {
      bf16x8 bf[8];
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) bf[kk] = row_frag(tb + J * kTile32, rp, kk);
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) af[1][kk] = row_frag(ta + kTile32, rp, kk);
      slot_end();
      f32x16 s[2];
      if (wave == 0)
        tile_product(s, bf, af[0]);
      else
        tile_product(s, bf, af[1]);
      settle(s[0], s[1]);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float f[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) f[r] = (s[0][8 * x + r] + s[1][8 * x + r]) * dec[8 * x + r];
        pf[wave][x][lane] = pack_bf16x8(f);
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) af[1][kk] = row_frag(ta + kTile32, rp, kk);
    }
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) cf[ks] = col_frag(tc + c_place, ks, wave);
    // y^T = S^T a^T, each row's weight on its lane
    f32x16 y[2];
    bf16x8 sf[8];
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) sf[kk] = operand8(st.s[kk >> 1], kk & 1);
    hold_in_vgprs(sf);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      if (kk == 0) {
        score_first(y[0], sf[kk], af[0][kk]);
        score_first(y[1], sf[kk], af[1][kk]);
      } else {
        score(y[0], sf[kk], af[0][kk]);
        score(y[1], sf[kk], af[1][kk]);
      }
    }
    settle(y[0], y[1]);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      y[0][r] *= win[0];
      y[1][r] *= win[1];
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    bf16x8 pt[3][2];
#pragma unroll
    for (int t = 0; t < 3; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) pt[t][x] = __builtin_bit_cast(bf16x8, pf[t][x][lane]);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      score(y[0], cf[x], pt[0][x]);
      score(y[1], cf[x], pt[1][x]);
      score(y[1], cf[2 + x], pt[2][x]);
    }
    update_state<kExact>(st, fade, tb, cf, wt[m < kC && i > 0], place, hh);
#pragma unroll
    for (int i2 = 0; i2 < 2; ++i2) {
      const int j = row + 32 * i2 + l32;
      if (j < W.rows) {
        const int n = S.reverse ? W.len - 1 - j : j;
        const int64_t at = y0 + (int64_t)n * S.y_n + 32 * wave + 4 * hh;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (S.y_f32)
            *reinterpret_cast<float4*>(static_cast<float*>(S.y) + at + 8 * x) =
                make_float4(y[i2][4 * x], y[i2][4 * x + 1], y[i2][4 * x + 2], y[i2][4 * x + 3]);
          else
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(S.y) + at + 8 * x) =
                make_uint2(pack_bf16x2(y[i2][4 * x], y[i2][4 * x + 1]), pack_bf16x2(y[i2][4 * x + 2], y[i2][4 * x + 3]));
        }
      }
    }
  }
  copies_landed<0>();  // none is under way when the wave ends
  settle(st.s[0], st.s[1]);
  settle(st.s[2], st.s[3]);
  if (A.sh.nseg == 1 && S.state_out) store_state(st, S.state_out + (int64_t)slab * kStateElems, col, hh);
}

// Gradients of shared heads: the sum, in head order, of the group's fp32 parts,
// rounded once.  One thread per 16-byte chunk of a row.
__global__ __launch_bounds__(kThreads) void lin_group_sum_kernel(const float* __restrict__ part, uint16_t* out,
                                                                 int64_t sb, int64_t sh, int64_t sn, int64_t chunks,
                                                                 int H, int Hk, int N) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= chunks) return;
  const int cc = (int)(i & 15);
  const int64_t row = i >> 4;
  const int n = (int)(row % N);
  const int64_t bh = row / N;
  const int hk = (int)(bh % Hk), b = (int)(bh / Hk), per = H / Hk;
  float f[8] = {};
  for (int u = 0; u < per; ++u) {
    const float4* p = reinterpret_cast<const float4*>(part + ((((int64_t)b * H + hk * per + u) * N + n) * D + cc * 8));
    const float4 x = p[0], y = p[1];
    f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
    f[4] += y.x; f[5] += y.y; f[6] += y.z; f[7] += y.w;
  }
  *reinterpret_cast<uint4*>(out + b * sb + hk * sh + (int64_t)n * sn + cc * 8) = pack_bf16x8(f);
}

// One token for each request: the state is read, decayed, added to and written,
// and multiplied by q on the way.  Its bytes bound it (64 KB in and out against
// 66 kflop), so a workgroup takes a quarter of a state's columns, four 16-byte
// loads a thread all in flight.
//
// A slot below 0 is an empty place of the batch: its output is zero.  One past
// the pool, or one that an earlier request of the call has, gives NaN: two
// requests never write one state.
__global__ __launch_bounds__(kThreads) void lin_step_kernel(LinStep A) {
  __shared__ __attribute__((aligned(16))) float part[4][32];
  lds_poison(part, sizeof(part));
  lds_poison_done();
  const int id = blockIdx.x >> 2, quarter = blockIdx.x & 3;
  const int r = id / A.H, h = id - r * A.H;
  const int t = threadIdx.x, c4 = t & 7, grp = t >> 3;
  const int slot = A.slots ? A.slots[r] : r;
  bool bad = slot >= A.n_slots;
  if (A.slots && slot >= 0)
    for (int i = t; i < r; i += kThreads) bad |= A.slots[i] == slot;
  bad = __syncthreads_or(bad);
  uint16_t* out = A.out.p + r * A.out.sb + h * A.out.sh + 32 * quarter;
  if (bad || slot < 0) {
    if (t < 32) out[t] = bad ? 0x7FC0 : 0;
    return;
  }
  const int hk = h / (A.H / A.Hk);
  const uint16_t* q = A.q.p + r * A.q.sb + h * A.q.sh;
  const uint16_t* k = A.k.p + r * A.k.sb + hk * A.k.sh;
  const uint16_t* v = A.v.p + r * A.v.sb + hk * A.v.sh + 32 * quarter + 4 * c4;
  float4* s = reinterpret_cast<float4*>(A.state + ((int64_t)slot * A.H + h) * kStateElems + 32 * quarter) + c4;
  float4 x[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) x[u] = s[(grp + 32 * u) * (D / 4)];
  const float decay = __builtin_amdgcn_exp2f(decay_log2(A.log_decay, h));
  auto f = [](uint16_t w) { return __uint_as_float((uint32_t)w << 16); };
  const float4 vv = make_float4(f(v[0]), f(v[1]), f(v[2]), f(v[3]));
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const float kk = f(k[grp + 32 * u]), qq = f(q[grp + 32 * u]);
    x[u].x = __builtin_fmaf(x[u].x, decay, kk * vv.x);
    x[u].y = __builtin_fmaf(x[u].y, decay, kk * vv.y);
    x[u].z = __builtin_fmaf(x[u].z, decay, kk * vv.z);
    x[u].w = __builtin_fmaf(x[u].w, decay, kk * vv.w);
    s[(grp + 32 * u) * (D / 4)] = x[u];
    o.x = __builtin_fmaf(qq, x[u].x, o.x);
    o.y = __builtin_fmaf(qq, x[u].y, o.y);
    o.z = __builtin_fmaf(qq, x[u].z, o.z);
    o.w = __builtin_fmaf(qq, x[u].w, o.w);
  }
  // the wave's eight rows groups, then the four waves'
#pragma unroll
  for (int m = 8; m < 64; m <<= 1) {
    o.x += __shfl_xor(o.x, m);
    o.y += __shfl_xor(o.y, m);
    o.z += __shfl_xor(o.z, m);
    o.w += __shfl_xor(o.w, m);
  }
  if ((t & 63) < 8) *reinterpret_cast<float4*>(&part[t >> 6][4 * c4]) = o;
  __syncthreads();
  if (t < 16) {
    const float a = part[0][2 * t] + part[1][2 * t] + part[2][2 * t] + part[3][2 * t];
    const float b = part[0][2 * t + 1] + part[1][2 * t + 1] + part[2][2 * t + 1] + part[3][2 * t + 1];
    reinterpret_cast<uint32_t*>(out)[t] = pack_bf16x2(A.scale * a, A.scale * b);
  }
}

// The state pass and the join where there are several segments, then the scans.
hipError_t launch_scans(const StateArgs& st, const ScanArgs& sc, int64_t slabs, bool exact_states, bool exact_scan,
                        hipStream_t stream) {
  const unsigned wgs = (unsigned)(slabs * sc.sh.nseg);
  if (sc.sh.nseg > 1) {
    if (exact_states)
      hipLaunchKernelGGL(lin_state_kernel<true>, dim3(wgs * st.n), dim3(kThreads), 0, stream, st);
    else
      hipLaunchKernelGGL(lin_state_kernel<false>, dim3(wgs * st.n), dim3(kThreads), 0, stream, st);
    hipLaunchKernelGGL(lin_join_kernel, dim3((unsigned)(slabs * 16 * st.n)), dim3(kThreads), 0, stream, st);
  }
  if (exact_scan)
    hipLaunchKernelGGL(lin_scan_kernel<true>, dim3(wgs * sc.n), dim3(kThreads), 0, stream, sc);
  else
    hipLaunchKernelGGL(lin_scan_kernel<false>, dim3(wgs * sc.n), dim3(kThreads), 0, stream, sc);
  return hipGetLastError();
}

Shape shape_of(const float* log_decay, const int32_t* lens, int B, int H, int N) {
  const LinPlan plan = lin_plan((int64_t)B * H, N);
  return {log_decay, lens, H, N, plan.seg_rows, plan.nseg};
}

Scan scan_of(const Rows& a, int a_div, const Rows& b, int b_div, const Rows& c, int c_div, const Rows& y) {
  Scan s = {};
  s.a = a;
  s.b = b;
  s.c = c;
  s.a_div = a_div;
  s.b_div = b_div;
  s.c_div = c_div;
  s.y = y.p;
  s.y_b = y.sb;
  s.y_h = y.sh;
  s.y_n = y.sn;
  return s;
}

}  // namespace

LinPlan lin_plan(int64_t slabs, int N) {
  // one workgroup on each of the 256 CUs, in segments of at least 256 tokens
  const int chunks = (N + kC - 1) / kC;
  int64_t nseg = 256 / slabs;
  nseg = nseg < 1 ? 1 : nseg;
  const int most = (chunks + 3) / 4;
  if (nseg > most) nseg = most;
  const int seg_chunks = (int)((chunks + nseg - 1) / nseg);
  return {seg_chunks * kC, (chunks + seg_chunks - 1) / seg_chunks};
}

size_t lin_states_bytes(int64_t slabs, int N) {
  const LinPlan p = lin_plan(slabs, N);
  return p.nseg > 1 ? (size_t)slabs * p.nseg * kStateElems * sizeof(float) : 0;
}

hipError_t launch_lin_fwd(const LinFwd& a, hipStream_t stream) {
  const int per = a.H / a.Hk;
  ScanArgs sc = {};
  sc.sh = shape_of(a.log_decay, a.lens, a.B, a.H, a.N);
  sc.n = 1;
  Scan& s = sc.scan[0];
  s = scan_of(a.q, 1, a.k, per, a.v, per, a.out);
  s.state_in = a.state_in;
  s.state_out = a.state_out;
  s.before = a.states;
  s.p = s.r = a.scale;
  s.u = 1.0f;
  s.off = 1;
  StateArgs st = {};
  st.sh = sc.sh;
  st.n = 1;
  st.st[0] = {a.k, a.v, per, per, a.state_in, 0, a.state_out, a.states, nullptr, 1.0f, 1, 0};
  const bool exact = a.state_out != nullptr;
  return launch_scans(st, sc, (int64_t)a.B * a.H, exact, exact && sc.sh.nseg == 1, stream);
}

// The three gradients in one launch (dq forwards; dk and dv backwards, side by
// side, so that the second to read a row finds it in L2); the states of dk are
// those of dv transposed.
hipError_t launch_lin_bwd(const LinBwd& a, hipStream_t stream) {
  const int per = a.H / a.Hk;
  const int64_t slabs = (int64_t)a.B * a.H, elems = slabs * a.N * D;
  ScanArgs sc = {};
  sc.sh = shape_of(a.log_decay, a.lens, a.B, a.H, a.N);
  sc.n = 3;
  const int64_t sec = slabs * sc.sh.nseg * kStateElems;  // floats of the segments' states
  sc.scan[0] = scan_of(a.dout, 1, a.v, per, a.k, per, a.dq);
  sc.scan[1] = scan_of(a.v, per, a.dout, 1, a.q, 1, a.dk);
  sc.scan[2] = scan_of(a.k, per, a.q, 1, a.dout, 1, a.dv);
  for (int i = 0; i < 3; ++i) {
    Scan& s = sc.scan[i];
    s.before = a.states + i * sec;
    s.state_in = i == 0 ? a.state_in : a.dstate_in;
    s.state_t = i < 2;
    s.p = a.scale;
    s.r = i == 0 ? a.scale : 1.0f;
    s.u = i == 0 ? 1.0f : a.scale;
    s.off = i == 0;
    s.reverse = i > 0;
    s.zero_tail = 1;
    if (i > 0 && a.partial) {
      s.y = a.partial + (i - 1) * elems;
      s.y_f32 = 1;
      s.y_n = D;
      s.y_h = (int64_t)a.N * D;
      s.y_b = a.H * s.y_h;
    }
  }
  // (dk reads the state that dv's final one may be written over: not in one launch)
  const bool in_place = a.dstate_out && a.dstate_out == a.dstate_in && sc.sh.nseg == 1;
  sc.scan[2].state_out = a.dstate_out;
  StateArgs st = {};
  st.sh = sc.sh;
  st.n = 2;
  st.st[0] = {a.v, a.k, per, per, a.state_in, 1, nullptr, a.states, nullptr, 1.0f, 1, 0};
  st.st[1] = {a.q, a.dout, 1, 1, a.dstate_in, 0, a.dstate_out, a.states + 2 * sec, a.states + sec, a.scale, 0, 1};
  const bool exact = a.dstate_out != nullptr, exact_scan = exact && sc.sh.nseg == 1;
  hipError_t e;
  if (in_place) {
    ScanArgs last = sc;
    sc.n = 2;
    last.n = 1;
    last.scan[0] = sc.scan[2];
    e = launch_scans(st, sc, slabs, exact, false, stream);
    if (e == hipSuccess) e = launch_scans(st, last, slabs, exact, exact_scan, stream);
  } else {
    e = launch_scans(st, sc, slabs, exact, exact_scan, stream);
  }
  if (e != hipSuccess) return e;
  if (a.partial) {
    const int64_t chunks = (int64_t)a.B * a.Hk * a.N * (D / 8);
    for (int which = 0; which < 2; ++which) {
      const Rows& y = which ? a.dv : a.dk;
      hipLaunchKernelGGL(lin_group_sum_kernel, dim3((unsigned)((chunks + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                         stream, a.partial + which * elems, y.p, y.sb, y.sh, y.sn, chunks, a.H, a.Hk, a.N);
    }
  }
  return hipGetLastError();
}

hipError_t launch_lin_step(const LinStep& a, hipStream_t stream) {
  hipLaunchKernelGGL(lin_step_kernel, dim3((unsigned)((int64_t)a.R * a.H * 4)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sol
