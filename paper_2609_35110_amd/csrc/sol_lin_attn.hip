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

#include <algorithm>

#include "sol_ops.h"
#include "sol_tiles.h"

namespace sol {
namespace {

constexpr int kThreads = 256, kScanThreads = 512;
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
  const float* before;    // several segments: the states before them, [slab][segment][part 0][128][128]
  int before_t;           // .. held transposed
  float p, r, u;
  int off;
  int reverse;    // walk the tokens from the last one
  int zero_tail;  // write zeros to the rows behind the sequence (bf16)
};
// The states that segments add, found in one pass for the scans that need them,
// a segment in `parts` of its own where it takes as many to fill the CUs.
struct SegmentStates {
  Rows b, c;
  int b_div, c_div;
  const float* state_in;
  int state_t;
  float* state_out;
  float* local;       // in: what the parts add; out: the states before the segments, at their first parts
  float u;
  int off;
  int reverse;
};
struct Shape {
  const float* log_decay;
  const int32_t* lens;
  int B, H, N, seg_rows, nseg;
  int parts;  // of a segment, in the state pass
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
    for (int r = 0; r < 16; r += 4) {
      const int row = state_row(t, r, hh);  // (four consecutive ones)
      if (transposed) {
        const float4 x = *reinterpret_cast<const float4*>(p + col * D + row);
        st.s[t][r] = x.x;
        st.s[t][r + 1] = x.y;
        st.s[t][r + 2] = x.z;
        st.s[t][r + 3] = x.w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) st.s[t][r + i] = p[(row + i) * D + col];
      }
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
// do not drift over long sequences.  A weighted row of c enters as the sum of two
// bf16, its rounding and the rounding of the rest, 2^-17 together.
__device__ __forceinline__ void fade_state(f32x16& s, float fade, int r0, int n) {
#pragma unroll
  for (int r = r0; r < r0 + n; ++r) s[r] = __builtin_fmaf(s[r], -fade, s[r]);
}
// The weighted rows as MFMA operands, 16 rows (ks) at a time: two in use.
struct Weighted {
  bf16x8 hi[2], lo[2];
  uint32_t h[4], l[4];
  // quarter q of row group ks: two rows
  template <int ks, int q, int n>
  __device__ __forceinline__ void make(const bf16x8 (&cf)[n], const float (&w)[n][8]) {
    const uint4 four = __builtin_bit_cast(uint4, cf[ks]);
    const uint32_t x = q == 0 ? four.x : q == 1 ? four.y : q == 2 ? four.z : four.w;
    const float x0 = __uint_as_float(x << 16) * w[ks][2 * q], x1 = __uint_as_float(x & 0xffff0000u) * w[ks][2 * q + 1];
    h[q] = pack_bf16x2(x0, x1);
    l[q] = pack_bf16x2(x0 - __uint_as_float(h[q] << 16), x1 - __uint_as_float(h[q] & 0xffff0000u));
    if constexpr (q == 3) {
      hi[ks & 1] = __builtin_bit_cast(bf16x8, make_uint4(h[0], h[1], h[2], h[3]));
      asm volatile("" : "+v"(hi[ks & 1]));
      lo[ks & 1] = __builtin_bit_cast(bf16x8, make_uint4(l[0], l[1], l[2], l[3]));
      asm volatile("" : "+v"(lo[ks & 1]));
    } else {
      asm volatile("" : "+v"(h[q]));
    }
  }
};

// A value that all lanes hold, in a scalar register (a division leaves it in a
// vector one).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The walk of a workgroup over its segment's chunks: rows [row0, rows) of the
// sequence in walking order.
struct Walk {
  int b, h, seg, len, row0, rows, chunks;
  int64_t at;  // of the segment's state
  float g2;
};
__device__ __forceinline__ Walk make_walk(const Shape& s, int id, int nseg, int seg_rows) {
  Walk w;
  const int slab = uniform(id / nseg);
  w.seg = id - slab * nseg;
  if (s.lens) {  // sequences of different lengths take turns: an XCD has some of each
    w.h = uniform(slab / s.B);
    w.b = slab - w.h * s.B;
  } else {
    w.b = uniform(slab / s.H);
    w.h = slab - w.b * s.H;
  }
  w.at = (int64_t)(w.b * s.H + w.h) * nseg + w.seg;
  w.len = length_of(s, w.b);
  w.row0 = w.seg * seg_rows;
  w.rows = min(w.row0 + seg_rows, w.len);
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

__device__ __forceinline__ float fade_of(float g2, int m) { return -expm1f(g2 * 0.693147180559945309f * (float)m); }

// w_j = u e^{g(m - off - j)} of this lane's rows in the transpose reads from row
// 16 ks0 on, in their order, for the m rows of a chunk, 0 past them.
template <int n>
__device__ __forceinline__ void row_weights(float (&w)[n][8], int ks0, float u, int off, float g2, int m, int hh) {
#pragma unroll
  for (int ks = 0; ks < n; ++ks)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = 16 * (ks0 + ks) + 4 * hh + (i & 3) + 8 * (i >> 2);
      w[ks][i] = j < m ? u * __builtin_amdgcn_exp2f(g2 * (float)max(m - off - j, 0)) : 0.0f;
    }
}
constexpr int kAhead = 6;  // operand reads on their way in the slots of a chunk

// The states that segments add, from zero: one pass over b and c, 128 rows a
// turn.  Eight waves, two a SIMD (one hides the other's waits): 32 columns of the
// state and one half of the turn's rows each, the halves' states added up at the
// end.
//
// Bound by its bytes when they come from HBM: 111,600 tokens x 40 heads 420 to 440
// us, 4.4 to 4.6 TB/s (370 us where the rows' second part is left out, which costs
// the states half their bits); 12,480 x 24 from the caches 34 us, 5.0 TB/s.  One wave
// a SIMD, 64 rows a turn, took 507 and 37.  Every row is read, those of a fast head
// too that leave nothing at the segment's end.
constexpr int kStateRows = 2 * kC;
__global__ __launch_bounds__(kScanThreads, 2) void lin_state_kernel(StateArgs A) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2][2][2][kTile];  // ring of two; b, c; halves
  lds_poison(lds, sizeof(lds));
  lds_poison_done();
  const int all = xcd_local_id(blockIdx.x, gridDim.x);
  const int id = uniform(all / A.n);
  const SegmentStates S = A.st[all - id * A.n];
  const Walk W = make_walk(A.sh, id, A.sh.nseg * A.sh.parts, A.sh.seg_rows / A.sh.parts);
  // the last segment's state is wanted by the final state alone
  if (W.seg >= (A.sh.nseg - 1) * A.sh.parts && !S.state_out) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hh = lane >> 5;
  const int wc = wave & 3, half = wave >> 2;  // columns, rows
  const int place = state_col_place(lane), c_place = col_place(lane);
  // waves 0 to 3 copy b, 4 to 7 c (past the last 64 rows those again: weight 0)
  const uint16_t* from = half ? slab_of(S.c, W, S.c_div) : slab_of(S.b, W, S.b_div);
  const int64_t sn = half ? S.c.sn : S.b.sn;
  const uint32_t at0 = lds_address(&lds[0][half][0][0]);
  auto copy = [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
      copy_chunk(at0 + (i & 1) * (4 * kTile) + x * kTile, from, sn, W, min(2 * i + x, W.chunks - 1), S.reverse, wc, lane);
  };
  State st{};
  const int turns = (W.chunks + 1) / 2;
  const int m0 = min(kStateRows, W.rows - W.row0);
  float fade = fade_of(W.g2, m0), w[4][8];
  row_weights(w, 4 * half, S.u, S.off, W.g2, m0, hh);
  all_landed();
  if (turns > 0) copy(0);
  for (int i = 0; i < turns; ++i) {
    const int m = min(kStateRows, W.rows - W.row0 - i * kStateRows);
    if (m < kStateRows && i > 0) {  // the last turn's own
      int h = hh;  // (not computed ahead of the loop and kept)
      asm volatile("" : "+v"(h));
      row_weights(w, 4 * half, S.u, S.off, W.g2, m, h);
      fade = fade_of(W.g2, m);
    }
    copies_landed<0>();
    const uint8_t *tb = lds[i & 1][0][half] + place, *tc = lds[i & 1][1][half] + c_place;
    bf16x8 cf[4], ring[kAhead];
    auto read = [&](auto slot) __attribute__((always_inline)) {
      constexpr int f = decltype(slot)::value;
      if constexpr (f < 16) ring[f % kAhead] = col_frag(tb, f >> 2, f & 3);
    };
    cf[0] = col_frag(tc, 0, wc);
    each<0, kAhead>(read);
#pragma unroll
    for (int ks = 1; ks < 4; ++ks) cf[ks] = col_frag(tc, ks, wc);
    slot_end();
    if (i + 1 < turns) copy(i + 1);
    Weighted x;
    fade_state(st.s[0], fade, 0, 16);
    each<0, 4>([&](auto q) __attribute__((always_inline)) { x.make<0, decltype(q)::value>(cf, w); });
    slot_end();
    asm volatile("s_nop 1" : "+v"(st.s[0]));
    // slots of two MFMAs (the parts of c w): the next weighted rows, and in the
    // first three the decay of the next result
    each<0, 16>([&](auto slot) __attribute__((always_inline)) {
      constexpr int f = decltype(slot)::value, ks = f >> 2, t = f & 3;
      if constexpr (ks < 3) x.make<ks + 1, t>(cf, w);
      score(st.s[t], ring[f % kAhead], x.hi[ks & 1]);
      score(st.s[t], ring[f % kAhead], x.lo[ks & 1]);
      read(std::integral_constant<int, f + kAhead>{});
      if constexpr (f < 3) {
        fade_state(st.s[f + 1], fade, 0, 16);
        asm volatile("s_nop 1" : "+v"(st.s[f + 1]));
      }
      slot_end();
    });
    settle(st.s[0], st.s[1]);
    settle(st.s[2], st.s[3]);
  }
  // the halves' sum
  __syncthreads();
  f32x16* other = reinterpret_cast<f32x16*>(&lds[0][0][0][0]) + wc * 256 + lane;
  if (half)
#pragma unroll
    for (int t = 0; t < 4; ++t) other[64 * t] = st.s[t];
  __syncthreads();
  if (half) return;
#pragma unroll
  for (int t = 0; t < 4; ++t) st.s[t] += other[64 * t];
  store_state(st, S.local + W.at * kStateElems, 32 * wc + (lane & 31), hh);
}

// The states before each segment, from what their parts add: in place, one
// workgroup per slab and 1,024 of its state's values, eight parts' loads in
// flight.  Few bytes and one chain: 24 heads x 10 segments 8 us.
__global__ __launch_bounds__(kThreads) void lin_join_kernel(StateArgs A) {
  const SegmentStates& S = A.st[blockIdx.x % A.n];
  const int slab = blockIdx.x / A.n >> 4, part = (blockIdx.x / A.n) & 15;
  const int b = slab / A.sh.H, h = slab - b * A.sh.H;
  const int len = length_of(A.sh, b), parts = A.sh.nseg * A.sh.parts, rows = A.sh.seg_rows / A.sh.parts;
  const float g2 = decay_log2(A.sh.log_decay, h);
  const int e = part * 1024 + threadIdx.x * 4, row = e >> 7, col = e & 127;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (S.state_in) {
    const float* p = S.state_in + (int64_t)slab * kStateElems;
    s = S.state_t ? make_float4(p[col * D + row], p[(col + 1) * D + row], p[(col + 2) * D + row], p[(col + 3) * D + row])
                  : *reinterpret_cast<const float4*>(p + e);
  }
  float* seg = S.local + (int64_t)slab * parts * kStateElems;
  const float whole = fade_of(g2, rows);
  const int last = S.state_out ? parts : parts - A.sh.parts;  // parts whose own state was found
  constexpr int kBatch = 8;
  for (int i0 = 0; i0 < parts; i0 += kBatch) {
    float4 x[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i0 + u < last) x[u] = *reinterpret_cast<const float4*>(seg + (int64_t)(i0 + u) * kStateElems + e);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int i = i0 + u;
      if (i < parts) {
        if (i % A.sh.parts == 0) *reinterpret_cast<float4*>(seg + (int64_t)i * kStateElems + e) = s;
        const int m = min(max(len - i * rows, 0), rows);
        const float fade = m == rows ? whole : fade_of(g2, m);
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

// y over a segment.  Eight waves, two a SIMD: four keep the state, four feed them.
//
// Waves 0 to 3 own 32 columns each of the state and of y: the state stays in
// registers (64 a lane), where an MFMA leaves it and the next one takes it as an
// operand (rounded to bf16 there, as the C x C product is where c takes it, since y
// is a bf16 result: the roundings are of the same size, 0.0023 of y's norm together
// where y's own is 0.0017).  Waves 4 to 7 copy the chunks straight into LDS (a ring of
// three, two on their way) and find the three 32 x 32 tiles on and below the
// diagonal of the C x C product, which they pass on in the order the next
// product reads them, while the others multiply by the state.
//
// One chunk of the first four, a slot an MFMA with its operand read kAhead slots
// before and a share of the vector work:
//   16  y = a S        with S (1 - fade) for the update, and the first weighted c
//   32  S += b^T (c w) with the next weighted c; the C x C tiles arrive on the way
//    6  z = P c        after half of those; the others add y and z up
//
// Bound by its bytes where the chip is full: 111,600 tokens x 40 heads 1,030 to
// 1,070 us, 4.3 to 4.5 TB/s of a copy's 4.94; 12,480 x 24 69 us, 4.7.  One workgroup
// alone takes 1.9 us a chunk (four waves that did all of it, one after the other,
// 2.75).  The gradients' three scans of 12,480 x 24: 190 to 195 us for 0.76 GB past L2.
constexpr int kScanRing = 3;
__global__ __launch_bounds__(kScanThreads, 2) void lin_scan_kernel(ScanArgs A) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kScanRing][3][kTile];
  __shared__ __attribute__((aligned(16))) uint4 pf[3][2][64];  // tiles (0,0), (1,0), (1,1): 16 columns, lane
  lds_poison(lds, sizeof(lds));
  lds_poison(pf, sizeof(pf));
  lds_poison_done();
  const int all = xcd_local_id(blockIdx.x, gridDim.x);
  const int id = uniform(all / A.n);
  const Scan S = A.scan[all - id * A.n];
  const Walk W = make_walk(A.sh, id, A.sh.nseg, A.sh.seg_rows);
  const int slab = W.b * A.sh.H + W.h;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hh = lane >> 5, l32 = lane & 31;
  const int64_t y0 = W.b * S.y_b + W.h * S.y_h;

  if (S.zero_tail) {  // rows of this segment behind the sequence
    const int r = threadIdx.x >> 4, cc = threadIdx.x & 15;
    const int end = min(W.row0 + A.sh.seg_rows, A.sh.N);
    for (int i = max(W.row0, W.len) + r; i < end; i += kScanThreads / 16) {
      const int64_t at = y0 + (int64_t)i * S.y_n + cc * 8;
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(S.y) + at) = make_uint4(0, 0, 0, 0);
    }
  }
  if (W.chunks == 0) {  // (of a sequence without tokens, the first and last segment)
    if (A.sh.nseg == 1 && S.state_out)
      for (int e = threadIdx.x; e < kStateElems; e += kScanThreads)
        S.state_out[(int64_t)slab * kStateElems + e] =
            !S.state_in ? 0.0f : S.state_in[(int64_t)slab * kStateElems + (S.state_t ? (e & 127) * D + (e >> 7) : e)];
    return;
  }
  const RowPlace rp = row_place(lane);

  if (wave >= 4) {
    const int wv = wave - 4;
    const uint16_t *pa = slab_of(S.a, W, S.a_div), *pb = slab_of(S.b, W, S.b_div), *pc = slab_of(S.c, W, S.c_div);
    const uint32_t at0 = lds_address(&lds[0][0][0]);
    auto copy = [&](int i) __attribute__((always_inline)) {
      const uint32_t to = at0 + (i % kScanRing) * (3 * kTile);
      copy_chunk(to, pa, S.a.sn, W, i, S.reverse, wv, lane);
      copy_chunk(to + kTile, pb, S.b.sn, W, i, S.reverse, wv, lane);
      copy_chunk(to + 2 * kTile, pc, S.c.sn, W, i, S.reverse, wv, lane);
    };
    all_landed();
    copy(0);
    if (W.chunks > 1) copy(1);
    // this wave's tile of the C x C product: rows 32 I + .. of a, 32 J + .. of b,
    // held transposed (lane: row of a), and its weights
    const int I = wv == 0 ? 0 : 1, J = wv == 2 ? 1 : 0;
    float dec[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int gap = (32 * I + l32) - (32 * J + 8 * (r >> 2) + 4 * hh + (r & 3));
      dec[r] = gap >= 0 ? S.p * __builtin_amdgcn_exp2f(W.g2 * (float)gap) : 0.0f;
    }
    for (int i = 0; i < W.chunks; ++i) {
      if (i + 1 < W.chunks)
        copies_landed<3 * kChunkCopies>();
      else
        copies_landed<0>();
      if (wv < 3) {
        const uint8_t *ta = lds[i % kScanRing][0] + I * kTile32, *tb = lds[i % kScanRing][1] + J * kTile32;
        bf16x8 af[8], bf[8];
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
          af[kk] = row_frag(ta, rp, kk);
          bf[kk] = row_frag(tb, rp, kk);
        }
        slot_end();
        f32x16 s[2];
        tile_product(s, bf, af);
        settle(s[0], s[1]);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float f[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) f[r] = (s[0][8 * x + r] + s[1][8 * x + r]) * dec[8 * x + r];
          pf[wv][x][lane] = pack_bf16x8(f);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (i + 2 < W.chunks) copy(i + 2);
    }
    return;
  }

  const int col = 32 * wave + l32;
  const int place = state_col_place(lane), c_place = col_place(lane);
  State st{};
  if (A.sh.nseg > 1)
    load_state(st, S.before + W.at * A.sh.parts * kStateElems, S.before_t, col, hh);
  else if (S.state_in)
    load_state(st, S.state_in + (int64_t)slab * kStateElems, S.state_t, col, hh);
  const float win[2] = {S.r * __builtin_amdgcn_exp2f(W.g2 * (float)(l32 + S.off)),
                        S.r * __builtin_amdgcn_exp2f(W.g2 * (float)(32 + l32 + S.off))};
  float fade = fade_of(W.g2, min(kC, W.rows - W.row0));
  float w[4][8];
  row_weights(w, 0, S.u, S.off, W.g2, min(kC, W.rows - W.row0), hh);
  all_landed();
  for (int i = 0; i < W.chunks; ++i) {
    const int row = W.row0 + i * kC, m = min(kC, W.rows - row);
    if (m < kC && i > 0) {  // the last chunk's own
      int half = hh;  // (not computed ahead of the loop and kept)
      asm volatile("" : "+v"(half));
      row_weights(w, 0, S.u, S.off, W.g2, m, half);
      fade = fade_of(W.g2, m);
    }
    bf16x8 sf[8];
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) sf[kk] = operand8(st.s[kk >> 1], kk & 1);
    hold_in_vgprs(sf);
    asm volatile("s_barrier" ::: "memory");
    const uint8_t *ta = lds[i % kScanRing][0], *tb = lds[i % kScanRing][1] + place, *tc = lds[i % kScanRing][2] + c_place;
    f32x16 y[2], z[2];
    bf16x8 ring[kAhead], cf[4], pt[3][2];
    Weighted x;
    uint32_t pk[8];
    auto read = [&](auto slot) __attribute__((always_inline)) {
      constexpr int f = decltype(slot)::value;
      if constexpr (f < 16)
        ring[f % kAhead] = row_frag(ta + (f & 1) * kTile32, rp, f >> 1);
      else if constexpr (f < 32)
        ring[f % kAhead] = col_frag(tb, (f - 16) >> 2, f & 3);
    };
    auto update = [&](auto slot) __attribute__((always_inline)) {
      constexpr int f = decltype(slot)::value, ks = (f - 16) >> 2, t = f & 3;
      if constexpr (ks < 3) x.make<ks + 1, t>(cf, w);
      score(st.s[t], ring[f % kAhead], x.hi[ks & 1]);
      score(st.s[t], ring[f % kAhead], x.lo[ks & 1]);
      read(std::integral_constant<int, f + kAhead>{});
      slot_end();
      if constexpr (f >= 24) {  // four rows' worth of y and z
        constexpr int o = (f - 24) >> 2, q = f & 3;
#pragma unroll
        for (int r = 4 * q; r < 4 * q + 4; ++r) y[o][r] = __builtin_fmaf(y[o][r], win[o], z[o][r]);
        pk[2 * q] = pack_bf16x2(y[o][4 * q], y[o][4 * q + 1]);
        pk[2 * q + 1] = pack_bf16x2(y[o][4 * q + 2], y[o][4 * q + 3]);
        asm volatile("" : "+v"(pk[2 * q]), "+v"(pk[2 * q + 1]));
      }
      slot_end();
    };
    auto store = [&](int o) __attribute__((always_inline)) {
      int j = row + 32 * o + l32;
      asm volatile("" : "+v"(j));
      const int n = S.reverse ? W.len - 1 - j : j;
      const int64_t at = y0 + (int64_t)n * S.y_n + 32 * wave;
      if (S.y_f32) {
        float4* p = reinterpret_cast<float4*>(static_cast<float*>(S.y) + at + 4 * hh);
        if (j < W.rows)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            p[2 * x] = make_float4(y[o][4 * x], y[o][4 * x + 1], y[o][4 * x + 2], y[o][4 * x + 3]);
      } else {  // eight columns a lane: the halves of the wave exchange four
#pragma unroll
        for (int x = 0; x < 4; x += 2)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const auto both = __builtin_amdgcn_permlane32_swap(pk[2 * x + e], pk[2 * x + 2 + e], false, false);
            pk[2 * x + e] = both[0];
            pk[2 * x + 2 + e] = both[1];
          }
        uint4* p = reinterpret_cast<uint4*>(static_cast<uint16_t*>(S.y) + at + 8 * hh);
        if (j < W.rows) {
          p[0] = make_uint4(pk[0], pk[1], pk[2], pk[3]);
          p[2] = make_uint4(pk[4], pk[5], pk[6], pk[7]);
        }
      }
    };
    each<0, kAhead>(read);
    slot_end();
    each<0, 16>([&](auto slot) __attribute__((always_inline)) {
      constexpr int f = decltype(slot)::value, t = f >> 2;
      fade_state(st.s[t], fade, 4 * (f & 3), 4);
      if constexpr (f >= 12) x.make<0, f - 12>(cf, w);
      asm volatile("" : "+v"(st.s[t]));
      if constexpr (f < 2)
        score_first(y[f], sf[0], ring[f % kAhead]);
      else
        score(y[f & 1], sf[f >> 1], ring[f % kAhead]);
      if constexpr (f >= 4 && f < 8) cf[f - 4] = col_frag(tc, f - 4, wave);
      read(std::integral_constant<int, f + kAhead>{});
      slot_end();
    });
    each<16, 20>(update);
    asm volatile("s_barrier" ::: "memory");
#pragma unroll
    for (int t = 0; t < 3; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) pt[t][x] = __builtin_bit_cast(bf16x8, pf[t][x][lane]);
    slot_end();
    each<20, 24>(update);
    score_first(z[0], cf[0], pt[0][0]);
    score_first(z[1], cf[0], pt[1][0]);
    score(z[0], cf[1], pt[0][1]);
    score(z[1], cf[1], pt[1][1]);
    score(z[1], cf[2], pt[2][0]);
    score(z[1], cf[3], pt[2][1]);
    slot_end();
    each<24, 28>(update);
    store(0);
    each<28, 32>(update);
    store(1);
    settle(st.s[0], st.s[1]);
    settle(st.s[2], st.s[3]);
  }
  if (A.sh.nseg == 1 && S.state_out) store_state(st, S.state_out + (int64_t)slab * kStateElems, col, hh);
}

// Gradients of shared heads, dk's and dv's: the sum, in head order, of the
// group's fp32 parts, rounded once, and zeros behind the sequence (where the
// parts were not written).  One thread per 16-byte chunk of a row; its bytes bound
// it (4 x 2,047 tokens, 16 heads on 4: 16 us).
struct GroupSum {
  const float* part;  // dk's [B, H, N, 128], then dv's
  Rows y[2];
  const int32_t* lens;
  int B, H, Hk, N;
};
__global__ __launch_bounds__(kThreads) void lin_group_sum_kernel(GroupSum A) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int cc = (int)(i & 15);
  int64_t bh = (i >> 4) / A.N;
  const int n = (int)((i >> 4) - bh * A.N), per = A.H / A.Hk;
  const int64_t heads = (int64_t)A.B * A.Hk;
  if (bh >= 2 * heads) return;
  const int which = bh >= heads;
  bh -= which * heads;
  const int b = (int)(bh / A.Hk), hk = (int)(bh - (int64_t)b * A.Hk);
  float f[8] = {};
  if (!A.lens || n < A.lens[b]) {
    const float* p = A.part + ((((int64_t)which * A.B + b) * A.H + hk * per) * A.N + n) * D + cc * 8;
    for (int u = 0; u < per; ++u, p += (int64_t)A.N * D) {
      const float4 x = reinterpret_cast<const float4*>(p)[0], y = reinterpret_cast<const float4*>(p)[1];
      f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
      f[4] += y.x; f[5] += y.y; f[6] += y.z; f[7] += y.w;
    }
  }
  const Rows& y = A.y[which];
  *reinterpret_cast<uint4*>(y.p + b * y.sb + hk * y.sh + (int64_t)n * y.sn + cc * 8) = pack_bf16x8(f);
}

// One token for each request: the state is read, decayed, added to and written,
// and multiplied by q on the way.  Its bytes bound it (64 KB in and out against
// 66 kflop), so a workgroup takes a quarter of a state's columns, four 16-byte
// loads a thread all in flight: 10,240 states 270 to 280 us, 4.8 to 5.0 TB/s; 24 of
// them 4 us, a launch and a load's latency.
//
// The decay is taken off as a difference, as in the chunks' states (fade_state):
// a factor next to 1 rounds the same way for every token, by up to 2^-25 of the
// state each (g = -1e-6: the rate 1.3 % off).
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
  const float fade = fade_of(decay_log2(A.log_decay, h), 1);
  auto f = [](uint16_t w) { return __uint_as_float((uint32_t)w << 16); };
  const float4 vv = make_float4(f(v[0]), f(v[1]), f(v[2]), f(v[3]));
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const float kk = f(k[grp + 32 * u]), qq = f(q[grp + 32 * u]);
    x[u].x = __builtin_fmaf(kk, vv.x, __builtin_fmaf(x[u].x, -fade, x[u].x));
    x[u].y = __builtin_fmaf(kk, vv.y, __builtin_fmaf(x[u].y, -fade, x[u].y));
    x[u].z = __builtin_fmaf(kk, vv.z, __builtin_fmaf(x[u].z, -fade, x[u].z));
    x[u].w = __builtin_fmaf(kk, vv.w, __builtin_fmaf(x[u].w, -fade, x[u].w));
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
hipError_t launch_scans(const StateArgs& st, const ScanArgs& sc, int64_t slabs, hipStream_t stream) {
  const unsigned wgs = (unsigned)(slabs * sc.sh.nseg);
  if (sc.sh.nseg > 1) {
    hipLaunchKernelGGL(lin_state_kernel, dim3(wgs * sc.sh.parts * st.n), dim3(kScanThreads), 0, stream, st);
    hipLaunchKernelGGL(lin_join_kernel, dim3((unsigned)(slabs * 16 * st.n)), dim3(kThreads), 0, stream, st);
  }
  hipLaunchKernelGGL(lin_scan_kernel, dim3(wgs * sc.n), dim3(kScanThreads), 0, stream, sc);
  return hipGetLastError();
}

Shape shape_of(const float* log_decay, const int32_t* lens, int B, int H, int N, int scans) {
  const LinPlan plan = lin_plan((int64_t)B * H, N, scans);
  return {log_decay, lens, B, H, N, plan.seg_rows, plan.nseg, plan.parts};
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

// Sets of states: dq's and dv's (dk's are dv's, transposed), or the forward's.
static int lin_sets(int scans) { return scans > 1 ? 2 : 1; }

// Segments: as many as give each of the 256 CUs one workgroup of the launch's
// scans, of 256 tokens at least, where that is the faster way.  In times of a
// chunk (1.9 us), n segments take C / n of the scan, 0.75 as many of the state
// pass, and 7 + workgroups / 64 for two more launches and the states' bytes.
// Measured, in us, one segment against n: forward of 2 heads x 512 tokens 20
// against 27 (n = 2), x 1,024 35 against 28 (4); 8 heads x 4,096 125 against 37 (16);
// 24 heads x 1,024 35 against 35 (4), x 2,048 67 against 39 (8); 64 heads x 1,024 37
// against 43 (4), x 2,048 67 against 58 (4); 128 heads x 2,048 71 against 91 (2), x
// 12,480 509 against 474 (2).  Gradients of 8 heads x 4,096 127 against 47 (8), 24
// heads x 1,024 37 against 41 (3), x 2,048 67 against 57 (3; 76 in 8); 64 heads x
// 2,048 85 against 116 (2).
LinPlan lin_plan(int64_t slabs, int N, int scans) {
  const int chunks = (N + kC - 1) / kC, most = (chunks + 3) / 4;
  const LinPlan one = {chunks * kC, 1, 1};
  const int64_t wanted = std::min<int64_t>(256 / (slabs * scans), most);
  if (wanted < 2) return one;
  int seg_chunks = (int)((chunks + wanted - 1) / wanted);
  const int nseg = (chunks + seg_chunks - 1) / seg_chunks;
  const double split = 1.75 * seg_chunks + 7 + (double)(slabs * nseg) / 64;
  if (split >= chunks) return one;
  int parts = (int)std::min<int64_t>(256 / (slabs * lin_sets(scans) * (nseg - 1)), seg_chunks / 4);
  parts = std::max(parts, 1);
  seg_chunks = (seg_chunks + parts - 1) / parts * parts;
  return {seg_chunks * kC, (chunks + seg_chunks - 1) / seg_chunks, parts};
}

size_t lin_states_bytes(int64_t slabs, int N, int scans) {
  const LinPlan p = lin_plan(slabs, N, scans);
  return p.nseg > 1 ? (size_t)slabs * p.nseg * p.parts * lin_sets(scans) * kStateElems * sizeof(float) : 0;
}

hipError_t launch_lin_fwd(const LinFwd& a, hipStream_t stream) {
  const int per = a.H / a.Hk;
  ScanArgs sc = {};
  sc.n = 1;
  sc.sh = shape_of(a.log_decay, a.lens, a.B, a.H, a.N, sc.n);
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
  st.st[0] = {a.k, a.v, per, per, a.state_in, 0, a.state_out, a.states, 1.0f, 1, 0};
  return launch_scans(st, sc, (int64_t)a.B * a.H, stream);
}

// The three gradients in one launch (dq forwards; dk and dv backwards, side by
// side, so that the second to read a row finds it in L2); the states of dk are
// those of dv transposed.
hipError_t launch_lin_bwd(const LinBwd& a, hipStream_t stream) {
  const int per = a.H / a.Hk;
  const int64_t slabs = (int64_t)a.B * a.H, elems = slabs * a.N * D;
  ScanArgs sc = {};
  sc.n = kMaxScans;
  sc.sh = shape_of(a.log_decay, a.lens, a.B, a.H, a.N, sc.n);
  const int64_t sec = slabs * sc.sh.nseg * sc.sh.parts * kStateElems;  // floats of the parts' states
  sc.scan[0] = scan_of(a.dout, 1, a.v, per, a.k, per, a.dq);
  sc.scan[1] = scan_of(a.v, per, a.dout, 1, a.q, 1, a.dk);
  sc.scan[2] = scan_of(a.k, per, a.q, 1, a.dout, 1, a.dv);
  for (int i = 0; i < 3; ++i) {
    Scan& s = sc.scan[i];
    s.before = a.states + (i > 0) * sec;
    s.before_t = i == 1;
    s.state_in = i == 0 ? a.state_in : a.dstate_in;
    s.state_t = i < 2;
    s.p = a.scale;
    s.r = i == 0 ? a.scale : 1.0f;
    s.u = i == 0 ? 1.0f : a.scale;
    s.off = i == 0;
    s.reverse = i > 0;
    s.zero_tail = !(i > 0 && a.partial);
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
  st.st[0] = {a.v, a.k, per, per, a.state_in, 1, nullptr, a.states, 1.0f, 1, 0};
  st.st[1] = {a.q, a.dout, 1, 1, a.dstate_in, 0, a.dstate_out, a.states + sec, a.scale, 0, 1};
  hipError_t e;
  if (in_place) {
    ScanArgs last = sc;
    sc.n = 2;
    last.n = 1;
    last.scan[0] = sc.scan[2];
    e = launch_scans(st, sc, slabs, stream);
    if (e == hipSuccess) e = launch_scans(st, last, slabs, stream);
  } else {
    e = launch_scans(st, sc, slabs, stream);
  }
  if (e != hipSuccess) return e;
  if (a.partial) {
    const int64_t chunks = 2 * (int64_t)a.B * a.Hk * a.N * (D / 8);
    const GroupSum sum = {a.partial, {a.dk, a.dv}, a.lens, a.B, a.H, a.Hk, a.N};
    hipLaunchKernelGGL(lin_group_sum_kernel, dim3((unsigned)((chunks + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                       stream, sum);
  }
  return hipGetLastError();
}

hipError_t launch_lin_step(const LinStep& a, hipStream_t stream) {
  hipLaunchKernelGGL(lin_step_kernel, dim3((unsigned)((int64_t)a.R * a.H * 4)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sol
