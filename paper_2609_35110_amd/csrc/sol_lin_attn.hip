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
struct ScanArgs {
  const uint16_t *a, *b, *c;
  int64_t a_b, a_h, a_n, b_b, b_h, b_n, c_b, c_h, c_n;
  int a_div, b_div, c_div;  // head h of the scan reads head h / div
  void* y;                  // bf16, or fp32 when y_f32
  int64_t y_b, y_h, y_n;
  int y_f32;
  const float* log_decay;
  const float* state_in;  // the state before the first token of a segment
  int state_t;            // state_in is held transposed
  float* state_out;       // one segment only: the state after the last token
  float* states;          // [slab][segment][128][128]: local states out (state pass), states before in
  const int32_t* lens;
  int H, N, seg_rows, nseg;
  int reverse;    // walk the tokens from the last one
  int zero_tail;  // write zeros to the rows behind the sequence
  float p, r, u;
  int off;
};

__device__ __forceinline__ float decay_log2(const float* log_decay, int h) {
  // -inf (a head without memory) becomes a number whose multiple by 0 is 0
  return fmaxf(log_decay[h], -1e30f) * 1.44269504088896341f;
}

using Tile = Stage<kC, kThreads>;

// The wave's 32 columns of the state as four 32 x 32 MFMA results: s[t][r] of
// lane l is S[32t + 8(r/4) + 4(l/32) + r%4][32 wave + l%32].
struct State {
  f32x16 s[4];
};
__device__ __forceinline__ int state_row(int t, int r, int hh) { return 32 * t + 8 * (r >> 2) + 4 * hh + (r & 3); }

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

// S = (1 - fade) S + b^T (c w): the decay is taken off as a difference, so that
// its rounding is relative to what is lost and slow heads (e^{64 g} next to 1)
// do not drift over long sequences.  A weighted row of c enters as the sum of
// two bf16 (the rounding and the rounding of the rest, 2^-17 together): the
// state is an fp32 result of its own.
__device__ __forceinline__ void update_state(State& st, float fade, const uint16_t* tb, const bf16x8 (&cf)[4],
                                             const float* w, int tr_off, int hh) {
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.s[t][r] = __builtin_fmaf(st.s[t][r], -fade, st.s[t][r]);
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    const float4 w0 = *reinterpret_cast<const float4*>(w + 16 * ks + 4 * hh);
    const float4 w1 = *reinterpret_cast<const float4*>(w + 16 * ks + 8 + 4 * hh);
    float x[8], rest[8];
    unpack_bf16x8(__builtin_bit_cast(uint4, cf[ks]), x);
    x[0] *= w0.x; x[1] *= w0.y; x[2] *= w0.z; x[3] *= w0.w;
    x[4] *= w1.x; x[5] *= w1.y; x[6] *= w1.z; x[7] *= w1.w;
    const uint4 hi = pack_bf16x8(x);
    unpack_bf16x8(hi, rest);
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = x[i] - rest[i];
    const uint4 lo = pack_bf16x8(rest);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bf16x8 bt = column8(tb + 16 * ks * kStride + 32 * t + tr_off);
      st.s[t] = mfma(bt, __builtin_bit_cast(bf16x8, hi), st.s[t]);
      st.s[t] = mfma(bt, __builtin_bit_cast(bf16x8, lo), st.s[t]);
    }
  }
}

// What a workgroup of either pass finds out first: its slab, its rows and its
// weights.
struct Walk {
  int b, h, seg, len, row0, rows;  // rows [row0, rows) of the (reversed) sequence
  const uint16_t *a, *bb, *c;
  int64_t an, bn, cn;
  float g2;
};
__device__ __forceinline__ Walk make_walk(const ScanArgs& A, int id) {
  Walk w;
  const int slab = id / A.nseg;
  w.seg = id - slab * A.nseg;
  w.b = slab / A.H;
  w.h = slab - w.b * A.H;
  w.len = A.lens ? min(max(A.lens[w.b], 0), A.N) : A.N;
  w.row0 = w.seg * A.seg_rows;
  w.rows = min(w.row0 + A.seg_rows, w.len);
  w.a = A.a + w.b * A.a_b + (w.h / A.a_div) * A.a_h;
  w.bb = A.b + w.b * A.b_b + (w.h / A.b_div) * A.b_h;
  w.c = A.c + w.b * A.c_b + (w.h / A.c_div) * A.c_h;
  w.an = A.a_n;
  w.bn = A.b_n;
  w.cn = A.c_n;
  if (A.reverse && w.len > 0) {
    w.a += (int64_t)(w.len - 1) * w.an;
    w.bb += (int64_t)(w.len - 1) * w.bn;
    w.c += (int64_t)(w.len - 1) * w.cn;
    w.an = -w.an;
    w.bn = -w.bn;
    w.cn = -w.cn;
  }
  w.g2 = decay_log2(A.log_decay, w.h);
  return w;
}

// w[j] = u e^{g(m - off - j)} for the m rows of a chunk (rows past them are zero).
__device__ __forceinline__ void fill_weights(float* w, const ScanArgs& A, float g2, int m) {
  if (threadIdx.x < kC) w[threadIdx.x] = A.u * __builtin_amdgcn_exp2f(g2 * (float)max(m - A.off - (int)threadIdx.x, 0));
}
__device__ __forceinline__ float fade_of(float g2, int m) { return -expm1f(g2 * 0.693147180559945309f * (float)m); }

// The state that a segment adds, from zero: one pass over b and c.
__global__ __launch_bounds__(kThreads, 2) void lin_state_kernel(ScanArgs A) {
  __shared__ __attribute__((aligned(16))) uint16_t tb[kC * kStride], tc[kC * kStride];
  __shared__ __attribute__((aligned(16))) float wt[kC];
  lds_poison(tb, sizeof(tb));
  lds_poison(tc, sizeof(tc));
  lds_poison(wt, sizeof(wt));
  lds_poison_done();
  const int id = xcd_local_id(blockIdx.x, gridDim.x);
  const Walk W = make_walk(A, id);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, hh = lane >> 5, l32 = lane & 31;
  const int tr_off = column_offset(lane);
  State st{};
  Tile sb, sc;
  sb.load(W.bb, W.bn, W.row0, W.rows, threadIdx.x);
  sc.load(W.c, W.cn, W.row0, W.rows, threadIdx.x);
  for (int row = W.row0; row < W.rows; row += kC) {
    const int m = min(kC, W.rows - row);
    sb.store(tb, threadIdx.x);
    sc.store(tc, threadIdx.x);
    if (row == W.row0 || m < kC) fill_weights(wt, A, W.g2, m);
    __syncthreads();
    sb.load(W.bb, W.bn, row + kC, W.rows, threadIdx.x);
    sc.load(W.c, W.cn, row + kC, W.rows, threadIdx.x);
    bf16x8 cf[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) cf[ks] = column8(tc + 16 * ks * kStride + 32 * wave + tr_off);
    update_state(st, fade_of(W.g2, m), tb, cf, wt, tr_off, hh);
    __syncthreads();
  }
  store_state(st, A.states + (int64_t)id * kStateElems, 32 * wave + l32, hh);
}

// The states before each segment, from the segments' own: in place, one
// workgroup per slab and 1,024 of its state's values.
__global__ __launch_bounds__(kThreads) void lin_join_kernel(ScanArgs A) {
  const int slab = blockIdx.x >> 4, part = blockIdx.x & 15;
  const int b = slab / A.H, h = slab - b * A.H;
  const int len = A.lens ? min(max(A.lens[b], 0), A.N) : A.N;
  const float g2 = decay_log2(A.log_decay, h);
  const int e = part * 1024 + threadIdx.x * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (A.state_in) {
    const float* p = A.state_in + (int64_t)slab * kStateElems;
    if (A.state_t) {
      const int row = e >> 7, col = e & 127;
      s = make_float4(p[col * D + row], p[(col + 1) * D + row], p[(col + 2) * D + row], p[(col + 3) * D + row]);
    } else {
      s = *reinterpret_cast<const float4*>(p + e);
    }
  }
  float4* seg = reinterpret_cast<float4*>(A.states + (int64_t)slab * A.nseg * kStateElems + e);
  float4 x = seg[0];
  for (int i = 0; i < A.nseg; ++i) {
    const float4 next = seg[(int64_t)min(i + 1, A.nseg - 1) * (kStateElems / 4)];
    seg[(int64_t)i * (kStateElems / 4)] = s;
    const float fade = fade_of(g2, min(max(len - i * A.seg_rows, 0), A.seg_rows));
    s.x = __builtin_fmaf(s.x, -fade, s.x) + x.x;
    s.y = __builtin_fmaf(s.y, -fade, s.y) + x.y;
    s.z = __builtin_fmaf(s.z, -fade, s.z) + x.z;
    s.w = __builtin_fmaf(s.w, -fade, s.w) + x.w;
    x = next;
  }
  if (A.state_out) *reinterpret_cast<float4*>(A.state_out + (int64_t)slab * kStateElems + e) = s;
}

// y over a segment.  A wave owns 32 columns of the state and of y: the state
// stays in its registers (64 a lane), where an MFMA leaves it and the next one
// takes it as an operand (rounded to bf16 there, as y is a bf16 result: both
// roundings are of the same size).  The C x C products are shared: waves 0 to 2
// find the three 32 x 32 tiles on and below the diagonal, and pass them round
// in the order the next product reads them.
__global__ __launch_bounds__(kThreads, 2) void lin_scan_kernel(ScanArgs A) {
  __shared__ __attribute__((aligned(16))) uint16_t ta[kC * kStride], tb[kC * kStride], tc[kC * kStride];
  __shared__ __attribute__((aligned(16))) uint4 pf[3][2][64];  // tiles (0,0), (1,0), (1,1): 16 columns, lane
  __shared__ __attribute__((aligned(16))) float wt[kC];
  lds_poison(ta, sizeof(ta));
  lds_poison(tb, sizeof(tb));
  lds_poison(tc, sizeof(tc));
  lds_poison(pf, sizeof(pf));
  lds_poison(wt, sizeof(wt));
  lds_poison_done();
  const int id = xcd_local_id(blockIdx.x, gridDim.x);
  const Walk W = make_walk(A, id);
  const int slab = W.b * A.H + W.h;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, hh = lane >> 5, l32 = lane & 31;
  const int tr_off = column_offset(lane);
  const int col = 32 * wave + l32;

  if (A.zero_tail) {  // rows of this segment behind the sequence
    const int r = threadIdx.x >> 4, cc = threadIdx.x & 15;
    const int end = min(W.row0 + A.seg_rows, A.N);
    for (int i = max(W.row0, W.len) + r; i < end; i += 16) {
      const int64_t at = W.b * A.y_b + W.h * A.y_h + (int64_t)i * A.y_n + cc * 8;
      if (A.y_f32) {
        float4* y = reinterpret_cast<float4*>(static_cast<float*>(A.y) + at);
        y[0] = y[1] = make_float4(0.f, 0.f, 0.f, 0.f);
      } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(A.y) + at) = make_uint4(0, 0, 0, 0);
      }
    }
  }

  State st{};
  if (A.nseg > 1)
    load_state(st, A.states + (int64_t)id * kStateElems, false, col, hh);
  else if (A.state_in)
    load_state(st, A.state_in + (int64_t)slab * kStateElems, A.state_t, col, hh);

  // this wave's tile of the C x C product: rows 32 I + .. of a, 32 J + .. of b,
  // held transposed (lane: row of a), and its weights
  const int I = wave == 0 ? 0 : 1, J = wave == 2 ? 1 : 0;
  float dec[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int gap = (32 * I + l32) - (32 * J + 8 * (r >> 2) + 4 * hh + (r & 3));
    dec[r] = gap >= 0 ? A.p * __builtin_amdgcn_exp2f(W.g2 * (float)gap) : 0.0f;
  }
  const float win[2] = {A.r * __builtin_amdgcn_exp2f(W.g2 * (float)(l32 + A.off)),
                        A.r * __builtin_amdgcn_exp2f(W.g2 * (float)(32 + l32 + A.off))};

  Tile sa, sb, sc;
  sa.load(W.a, W.an, W.row0, W.rows, threadIdx.x);
  sb.load(W.bb, W.bn, W.row0, W.rows, threadIdx.x);
  sc.load(W.c, W.cn, W.row0, W.rows, threadIdx.x);
  for (int row = W.row0; row < W.rows; row += kC) {
    const int m = min(kC, W.rows - row);
    sa.store(ta, threadIdx.x);
    sb.store(tb, threadIdx.x);
    sc.store(tc, threadIdx.x);
    if (row == W.row0 || m < kC) fill_weights(wt, A, W.g2, m);
    __syncthreads();
    sa.load(W.a, W.an, row + kC, W.rows, threadIdx.x);
    sb.load(W.bb, W.bn, row + kC, W.rows, threadIdx.x);
    sc.load(W.c, W.cn, row + kC, W.rows, threadIdx.x);
    if (wave < 3) {
      f32x16 s = {};
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) {
        s = mfma(row8(tb + 32 * J * kStride, lane, kk), row8(ta + 32 * I * kStride, lane, kk), s);
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = s[8 * x + i] * dec[8 * x + i];
        pf[wave][x][lane] = pack_bf16x8(f);
      }
    }
    // y^T = S^T a^T, each row's weight on its lane
    f32x16 y[2] = {};
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const bf16x8 sf = operand8(st.s[t], x);
#pragma unroll
        for (int i2 = 0; i2 < 2; ++i2) {
          const uint16_t* p = ta + (32 * i2 + l32) * kStride + 32 * t + 16 * x + 4 * hh;
          const uint2 lo = *reinterpret_cast<const uint2*>(p), hi = *reinterpret_cast<const uint2*>(p + 8);
          y[i2] = mfma(sf, __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y)), y[i2]);
        }
      }
#pragma unroll
    for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
      for (int r = 0; r < 16; ++r) y[i2][r] *= win[i2];
    bf16x8 cf[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) cf[ks] = column8(tc + 16 * ks * kStride + 32 * wave + tr_off);
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      y[0] = mfma(cf[x], __builtin_bit_cast(bf16x8, pf[0][x][lane]), y[0]);
      y[1] = mfma(cf[x], __builtin_bit_cast(bf16x8, pf[1][x][lane]), y[1]);
      y[1] = mfma(cf[2 + x], __builtin_bit_cast(bf16x8, pf[2][x][lane]), y[1]);
    }
#pragma unroll
    for (int i2 = 0; i2 < 2; ++i2) {
      const int i = row + 32 * i2 + l32;
      if (i < W.rows) {
        const int n = A.reverse ? W.len - 1 - i : i;
        const int64_t at = W.b * A.y_b + W.h * A.y_h + (int64_t)n * A.y_n + 32 * wave + 4 * hh;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (A.y_f32)
            *reinterpret_cast<float4*>(static_cast<float*>(A.y) + at + 8 * x) =
                make_float4(y[i2][4 * x], y[i2][4 * x + 1], y[i2][4 * x + 2], y[i2][4 * x + 3]);
          else
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(A.y) + at + 8 * x) =
                make_uint2(pack_bf16x2(y[i2][4 * x], y[i2][4 * x + 1]), pack_bf16x2(y[i2][4 * x + 2], y[i2][4 * x + 3]));
        }
      }
    }
    update_state(st, fade_of(W.g2, m), tb, cf, wt, tr_off, hh);
    __syncthreads();
  }
  if (A.nseg == 1 && A.state_out) store_state(st, A.state_out + (int64_t)slab * kStateElems, col, hh);
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

// The state pass and the join where there are several segments, then the scan.
hipError_t launch_scan(ScanArgs& A, int64_t slabs, hipStream_t stream) {
  const LinPlan plan = lin_plan(slabs, A.N);
  A.seg_rows = plan.seg_rows;
  A.nseg = plan.nseg;
  const unsigned wgs = (unsigned)(slabs * plan.nseg);
  if (plan.nseg > 1) {
    hipLaunchKernelGGL(lin_state_kernel, dim3(wgs), dim3(kThreads), 0, stream, A);
    hipLaunchKernelGGL(lin_join_kernel, dim3((unsigned)(slabs * 16)), dim3(kThreads), 0, stream, A);
  }
  hipLaunchKernelGGL(lin_scan_kernel, dim3(wgs), dim3(kThreads), 0, stream, A);
  return hipGetLastError();
}

void set_rows(const uint16_t*& p, int64_t& sb, int64_t& sh, int64_t& sn, const Rows& r) {
  p = r.p;
  sb = r.sb;
  sh = r.sh;
  sn = r.sn;
}

ScanArgs scan_args(const Rows& a, int a_div, const Rows& b, int b_div, const Rows& c, int c_div, const float* log_decay,
                   const int32_t* lens, int H, int N, float* states) {
  ScanArgs A = {};
  set_rows(A.a, A.a_b, A.a_h, A.a_n, a);
  set_rows(A.b, A.b_b, A.b_h, A.b_n, b);
  set_rows(A.c, A.c_b, A.c_h, A.c_n, c);
  A.a_div = a_div;
  A.b_div = b_div;
  A.c_div = c_div;
  A.log_decay = log_decay;
  A.lens = lens;
  A.H = H;
  A.N = N;
  A.states = states;
  return A;
}

void set_out(ScanArgs& A, const Rows& y) {
  A.y = y.p;
  A.y_b = y.sb;
  A.y_h = y.sh;
  A.y_n = y.sn;
}

}  // namespace

LinPlan lin_plan(int64_t slabs, int N) {
  // two workgroups on each of the 256 CUs, in segments of at least 256 tokens
  const int chunks = (N + kC - 1) / kC;
  int64_t nseg = 512 / slabs;
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
  ScanArgs A = scan_args(a.q, 1, a.k, per, a.v, per, a.log_decay, a.lens, a.H, a.N, a.states);
  set_out(A, a.out);
  A.state_in = a.state_in;
  A.state_out = a.state_out;
  A.p = A.r = a.scale;
  A.u = 1.0f;
  A.off = 1;
  return launch_scan(A, (int64_t)a.B * a.H, stream);
}

hipError_t launch_lin_bwd(const LinBwd& a, hipStream_t stream) {
  const int per = a.H / a.Hk;
  const int64_t slabs = (int64_t)a.B * a.H;
  {
    ScanArgs A = scan_args(a.dout, 1, a.v, per, a.k, per, a.log_decay, a.lens, a.H, a.N, a.states);
    set_out(A, a.dq);
    A.state_in = a.state_in;
    A.state_t = 1;
    A.p = A.r = a.scale;
    A.u = 1.0f;
    A.off = 1;
    A.zero_tail = 1;
    const hipError_t e = launch_scan(A, slabs, stream);
    if (e != hipSuccess) return e;
  }
  // dk, then dv, whose state is the gradient of the initial state (and may be
  // written over the one that both read)
  for (int which = 0; which < 2; ++which) {
    ScanArgs A = which == 0 ? scan_args(a.v, per, a.dout, 1, a.q, 1, a.log_decay, a.lens, a.H, a.N, a.states)
                            : scan_args(a.k, per, a.q, 1, a.dout, 1, a.log_decay, a.lens, a.H, a.N, a.states);
    const Rows& y = which == 0 ? a.dk : a.dv;
    float* part = a.partial ? a.partial + which * slabs * a.N * D : nullptr;
    if (part) {
      A.y = part;
      A.y_f32 = 1;
      A.y_n = D;
      A.y_h = (int64_t)a.N * D;
      A.y_b = a.H * A.y_h;
    } else {
      set_out(A, y);
    }
    A.state_in = a.dstate_in;
    A.state_t = which == 0;
    A.state_out = which == 1 ? a.dstate_out : nullptr;
    A.p = A.u = a.scale;
    A.r = 1.0f;
    A.off = 0;
    A.reverse = 1;
    A.zero_tail = 1;
    hipError_t e = launch_scan(A, slabs, stream);
    if (e != hipSuccess) return e;
    if (part) {
      const int64_t chunks = (int64_t)a.B * a.Hk * a.N * (D / 8);
      hipLaunchKernelGGL(lin_group_sum_kernel, dim3((unsigned)((chunks + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                         stream, part, y.p, y.sb, y.sh, y.sn, chunks, a.H, a.Hk, a.N);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

hipError_t launch_lin_step(const LinStep& a, hipStream_t stream) {
  hipLaunchKernelGGL(lin_step_kernel, dim3((unsigned)((int64_t)a.R * a.H * 4)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sol
