// Queries and keys normalised and rotated at positions of their own
// (sol_qk_norm_rope, sol_qk_norm_rope_bwd):
//   y = R(pos) (gamma x r),   r = (mean x^2 + eps)^(-1/2),
// and with n = R(pos)^T dy, xh = x r, h = gamma n
//   dx = r (h - xh mean(h xh)),   dgamma = sum over the rows of n xh.
// Streaming kernels: 16 lanes hold a row, 16 rows of 16 tokens a workgroup and
// step; a thread keeps its token and its 8 dims through the heads that it walks,
// so that the position and its cosines and sines are found once for all of them.
#include <hip/hip_runtime.h>

#include "sol_cross.h"
#include "sol_device.h"

namespace sol {
namespace {

constexpr int kTokens = 16;  // of a workgroup's step

// A token, and how this thread's chunk cc of its rows turns: its first pair in the
// table, or not at all (a coordinate below 0, dims past the split, no positions).
struct Token {
  int b, n;
  bool inside;  // the sequence's own (and the batch's)
  bool bad;     // a coordinate past the table: the token's rows are NaN
  int pair;
};
constexpr int kStays = -1;
template <bool kRope>
__device__ __forceinline__ Token token_of(const NormRope& s, int64_t i, int cc) {
  Token t;
  t.b = (int)(i / s.N);
  t.n = (int)(i - (int64_t)t.b * s.N);
  t.inside = i < (int64_t)s.B * s.N && (s.lens == nullptr || t.n < min(max(s.lens[t.b], 0), s.N));
  t.bad = false;
  t.pair = kStays;
  if (kRope && t.inside) {
    const SeqGrid& g = s.g;
    const int32_t* p = s.pos + t.b * s.pos_sb + 3 * (int64_t)t.n;
    const int pt = p[0], ph = p[1], pw = p[2];
    // (an axis without dims has no coordinate)
    t.bad = (g.c_t > 0 && pt >= g.T) || (g.c_h > g.c_t && ph >= g.Hl) || (g.c_w > g.c_h && pw >= g.Wl);
    if (t.bad || cc >= g.c_w) return t;
    if (cc < g.c_t) t.pair = pt < 0 ? kStays : pt * g.s_t + 4 * cc;
    else if (cc < g.c_h) t.pair = ph < 0 ? kStays : g.tab_h + ph * g.s_h + 4 * (cc - g.c_t);
    else t.pair = pw < 0 ? kStays : g.tab_w + pw * g.s_w + 4 * (cc - g.c_h);
  }
  return t;
}
__device__ __forceinline__ RopeCS turns(const NormRope& s, const Token& t) {
  if (t.pair >= 0) return load_rope_cs(s.tab, tab_lo_plane(s.tab, s.g), t.pair);
  RopeCS cs;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    cs.c[u] = 1.0;
    cs.s[u] = 0.0;
  }
  return cs;
}
__device__ __forceinline__ uint4 nan_row() { return make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u); }
// (made where the compiler, which takes arithmetic to be free of NaN, does not see it)
__device__ __forceinline__ float nan_value() {
  float x;
  asm volatile("v_mov_b32 %0, 0x7fc00000" : "=v"(x));
  return x;
}

__device__ __forceinline__ uint16_t* row_at(const Rows& r, const Token& t, int h) {
  return r.p + t.b * r.sb + h * r.sh + (int64_t)t.n * r.sn;
}

// Heads [from, to) of the H + Hk of a token, q's first.
template <bool kRope>
__global__ __launch_bounds__(256) void norm_rope_fwd_kernel(NormRopeFwd A, int per_wg) {
  const NormRope& s = A.s;
  const int cc = threadIdx.x & 15;
  const Token t = token_of<kRope>(s, (int64_t)blockIdx.x * kTokens + (threadIdx.x >> 4), cc);
  if (!t.inside) return;  // whole rows: the lanes of a row leave together
  const RopeCS cs = kRope ? turns(s, t) : RopeCS{};
  float gq[8], gk[8];
  if (s.q_gamma) load_gamma(s.q_gamma, cc, gq);
  if (s.k_gamma) load_gamma(s.k_gamma, cc, gk);
  const int from = blockIdx.y * per_wg, to = min(from + per_wg, s.H + s.Hk);
  auto walk = [&](const Rows& x, const Rows& y, const float* gamma, const float (&gm)[8], int h0, int h1) {
    for (int h = h0; h < h1; ++h) {
      const uint4 v = *reinterpret_cast<const uint4*>(row_at(x, t, h) + 8 * cc);
      float f[8];
      if (gamma) norm_chunk(v, rms_inv(row_sumsq_lanes16(chunk_sumsq(v)), s.eps), gm, f);
      else unpack_bf16x8(v, f);
      uint4 out = gamma ? pack_bf16x8(f) : v;
      if (kRope && t.pair != kStays) out = rope_rotate(f, cs);
      *reinterpret_cast<uint4*>(row_at(y, t, h) + 8 * cc) = kRope && t.bad ? nan_row() : out;
    }
  };
  walk(A.q, A.q_out, s.q_gamma, gq, from, min(to, s.H));
  walk(A.k, A.k_out, s.k_gamma, gk, max(from - s.H, 0), to - s.H);
}

// R(pos)^T of a chunk, in fp32 with cosines and sines rounded to it (gradients are
// rounded to bf16 once, and sums of them are fp32: 2^-24 of a pair is far below either).
__device__ __forceinline__ void turn_back(float (&f)[8], const RopeCS& cs) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const float c = (float)cs.c[u], n = (float)cs.s[u], a = f[2 * u], b = f[2 * u + 1];
    f[2 * u] = __builtin_fmaf(a, c, b * n);
    f[2 * u + 1] = __builtin_fmaf(b, c, -(a * n));
  }
}

// The gradients: tiles of 16 tokens, every gridDim.x-th a workgroup, `per_wg` heads of
// each, the next head's rows on their way while one's are worked on; gamma's gradient
// is summed over a thread's rows, then over the workgroup's 16 tokens, then
// (norm_rope_gamma_kernel) over the workgroups.
template <bool kRope>
__global__ __launch_bounds__(256) void norm_rope_bwd_kernel(NormRopeBwd A, int per_wg) {
  __shared__ float sum[2][kTokens][D];
  lds_poison(sum, sizeof(sum));
  lds_poison_done();
  const NormRope& s = A.s;
  const int cc = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int from = blockIdx.y * per_wg, to = min(from + per_wg, s.H + s.Hk);
  float gq[8], gk[8], sq[8] = {}, sk[8] = {};
  if (s.q_gamma) load_gamma(s.q_gamma, cc, gq);
  if (s.k_gamma) load_gamma(s.k_gamma, cc, gk);
  const int64_t tokens = (int64_t)s.B * s.N, tiles = (tokens + kTokens - 1) / kTokens;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t i = tile * kTokens + r;
    if (i >= tokens) break;  // whole rows (a last tile's)
    const Token t = token_of<kRope>(s, i, cc);
    const RopeCS cs = kRope ? turns(s, t) : RopeCS{};
    if (kRope && t.bad)
      for (int e = 0; e < 8; ++e) sq[e] = sk[e] = nan_value();
    auto walk = [&](const Rows& dy, const Rows& x, const Rows& dx, const float* gamma, const float (&gm)[8], float (&sg)[8],
                    int h0, int h1) {
      if (h0 >= h1) return;
      if (!t.inside) {  // zero behind the sequence
        for (int h = h0; h < h1; ++h) *reinterpret_cast<uint4*>(row_at(dx, t, h) + 8 * cc) = make_uint4(0, 0, 0, 0);
        return;
      }
      auto load = [&](const Rows& z, int h) { return *reinterpret_cast<const uint4*>(row_at(z, t, min(h, h1 - 1)) + 8 * cc); };
      auto step = [&](int h, const uint4& y, const uint4& v) {
        float g[8];
        unpack_bf16x8(y, g);
        if (kRope) turn_back(g, cs);
        if (gamma) {
          const float inv = rms_inv(row_sumsq_lanes16(chunk_sumsq(v)), s.eps);
          float f[8], dot = 0.0f;
          unpack_bf16x8(v, f);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            f[e] *= inv;
            sg[e] = __builtin_fmaf(g[e], f[e], sg[e]);
            g[e] *= gm[e];
            dot = __builtin_fmaf(g[e], f[e], dot);
          }
          dot = row_sumsq_lanes16(dot) * (1.0f / D);
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = inv * __builtin_fmaf(-f[e], dot, g[e]);
        }
        *reinterpret_cast<uint4*>(row_at(dx, t, h) + 8 * cc) = kRope && t.bad ? nan_row() : pack_bf16x8(g);
      };
      // (two heads a trip: no load in flight moves between registers; past the last head it is read again)
      uint4 ya = load(dy, h0), va = gamma ? load(x, h0) : ya;
      for (int h = h0; h < h1; h += 2) {
        const uint4 yb = load(dy, h + 1), vb = gamma ? load(x, h + 1) : yb;
        step(h, ya, va);
        ya = load(dy, h + 2);
        va = gamma ? load(x, h + 2) : ya;
        if (h + 1 < h1) step(h + 1, yb, vb);
      }
    };
    walk(A.dq_out, A.q, A.dq, s.q_gamma, gq, sq, from, min(to, s.H));
    walk(A.dk_out, A.k, A.dk, s.k_gamma, gk, sk, max(from - s.H, 0), to - s.H);
  }
  if (A.partial == nullptr) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sum[0][r][8 * cc + e] = sq[e];
    sum[1][r][8 * cc + e] = sk[e];
  }
  __syncthreads();
  const int which = threadIdx.x >> 7, d = threadIdx.x & 127;
  float x = 0.0f;
#pragma unroll
  for (int u = 0; u < kTokens; ++u) x += sum[which][u][d];
  A.partial[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (2 * D) + threadIdx.x] = x;
}

// The workgroups' sums of gamma's gradients joined in one order, in 64 bits: 4 of the
// 256 columns a workgroup, 64 slices of the rows, the slices of a wave and then the waves.
constexpr int kGammaCols = 4, kGammaSlices = 256 / kGammaCols;
__global__ __launch_bounds__(256) void norm_rope_gamma_kernel(const float* __restrict__ partial, int n, float* dq_gamma,
                                                              float* dk_gamma) {
  __shared__ double sum[4][kGammaCols];
  lds_poison(sum, sizeof(sum));
  lds_poison_done();
  const int c = threadIdx.x % kGammaCols, slice = threadIdx.x / kGammaCols;
  const int col = blockIdx.x * kGammaCols + c;
  double x = 0.0;
#pragma unroll 8
  for (int i = slice; i < n; i += kGammaSlices) x += (double)partial[(int64_t)i * (2 * D) + col];
#pragma unroll
  for (int m = kGammaCols; m < 64; m <<= 1) x += __shfl_xor(x, m);
  if ((threadIdx.x & 63) < kGammaCols) sum[threadIdx.x >> 6][c] = x;
  __syncthreads();
  if (threadIdx.x >= kGammaCols) return;
  x = (sum[0][c] + sum[1][c]) + (sum[2][c] + sum[3][c]);
  float* to = col < D ? dq_gamma : dk_gamma;
  if (to) to[col % D] = (float)x;
}

}  // namespace

hipError_t launch_norm_rope_fwd(const NormRopeFwd& a, hipStream_t stream) {
  const NormRope& s = a.s;
  const int64_t tiles = ((int64_t)s.B * s.N + kTokens - 1) / kTokens;
  const int heads = s.H + s.Hk;
  // as many heads a workgroup as make eight workgroups a CU (of which it holds seven at once)
  int64_t per = tiles * heads / kStreamWgs;
  per = per < 1 ? 1 : per > heads ? heads : per;
  const int64_t groups = (heads + per - 1) / per;
  const auto kernel = s.pos ? norm_rope_fwd_kernel<true> : norm_rope_fwd_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)tiles, (unsigned)groups), dim3(256), 0, stream, a, (int)per);
  return hipGetLastError();
}

// Tiles of tokens a round, and parts of the heads, of the gradients' launch: eight
// workgroups a CU, of which its registers hold four at once (five without positions), in
// two rounds (512 tiles of 20 heads 25.8 us whole, 20.4 in four parts).
static void bwd_grid(int64_t tokens, int heads, int64_t* tiles, int* per) {
  const int64_t all = (tokens + kTokens - 1) / kTokens;
  *tiles = all < kStreamWgs ? all : kStreamWgs;
  const int64_t parts = kStreamWgs / *tiles;
  *per = (int)(parts >= heads ? 1 : (heads + parts - 1) / parts);
}
static int64_t bwd_workgroups(int64_t tokens, int heads) {
  int64_t tiles;
  int per;
  bwd_grid(tokens, heads, &tiles, &per);
  return tiles * ((heads + per - 1) / per);
}
size_t norm_rope_bwd_bytes(int64_t tokens, int heads) {
  return (size_t)bwd_workgroups(tokens, heads) * 2 * D * sizeof(float);
}

hipError_t launch_norm_rope_bwd(const NormRopeBwd& a, hipStream_t stream) {
  const NormRope& s = a.s;
  const int heads = s.H + s.Hk;
  int64_t tiles;
  int per;
  bwd_grid((int64_t)s.B * s.N, heads, &tiles, &per);
  const auto kernel = s.pos ? norm_rope_bwd_kernel<true> : norm_rope_bwd_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)tiles, (unsigned)((heads + per - 1) / per)), dim3(256), 0, stream, a, per);
  if (a.partial)
    hipLaunchKernelGGL(norm_rope_gamma_kernel, dim3(2 * D / kGammaCols), dim3(256), 0, stream, a.partial,
                       (int)bwd_workgroups((int64_t)s.B * s.N, heads), a.dq_gamma, a.dk_gamma);
  return hipGetLastError();
}

}  // namespace sol
