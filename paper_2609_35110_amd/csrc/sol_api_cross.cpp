// C ABI front end of the norm and rotation at given positions and of cross
// attention: argument validation (before any HIP call), launch and error mapping.
#include <cmath>

#include "sol_checks.h"
#include "sol_cross.h"

namespace {

constexpr int64_t kMaxTokens = ((int64_t)1 << 28) - 16;  // of a batch: a launch has 16 threads a token and fewer than 2^32
constexpr int kMaxHeads = (1 << 16) - 1;                 // of q and k: a head may be a workgroup of a grid's second axis

int check_norm_rope_sizes(int B, int H, int Hk, int N, int D) {
  if (B < 1 || H < 1 || Hk < 0 || N < 1)
    return fail(SOL_ERR_INVALID_ARG, "B, H, N must be >= 1 and Hk >= 0 (got %d, %d, %d, %d)", B, H, N, Hk);
  if (D != sol::kHeadDim) return fail(SOL_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", D);
  if (N > SOL_MAX_TOKENS) return fail(SOL_ERR_UNSUPPORTED, "N=%d exceeds %d", N, SOL_MAX_TOKENS);
  if ((int64_t)B * N > kMaxTokens) return fail(SOL_ERR_UNSUPPORTED, "B*N too large (at most 2^28 - 16)");
  if ((int64_t)H + Hk > kMaxHeads) return fail(SOL_ERR_UNSUPPORTED, "H + Hk too large (at most 2^16 - 1)");
  return SOL_OK;
}

// The table's sections: of a grid whose extents bound the coordinates, whatever
// the tokens are.
sol::SeqGrid sections(int T, int Hl, int Wl, int dt, int dh, int dw) {
  sol::SeqGrid g = {};
  g.T = T;
  g.Hl = Hl;
  g.Wl = Wl;
  g.c_t = dt / 8;
  g.c_h = g.c_t + dh / 8;
  g.c_w = g.c_h + dw / 8;
  g.s_t = dt / 2;
  g.s_h = dh / 2;
  g.s_w = dw / 2;
  g.tab_h = T * g.s_t;
  g.tab_w = g.tab_h + Hl * g.s_h;
  g.tab_pairs = g.tab_w + Wl * g.s_w;
  return g;
}

// Sizes, norm, positions and table of both directions of the norm and rotation.
int take_norm_rope(sol::NormRope* s, const float* q_gamma, const float* k_gamma, float eps, const int32_t* pos,
                   int64_t pos_stride_b, const float* tab, int T, int Hl, int Wl, int dt, int dh, int dw,
                   const int32_t* lens, int B, int H, int Hk, int N, int D) {
  SOL_TRY(check_norm_rope_sizes(B, H, Hk, N, D));
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(SOL_ERR_INVALID_ARG, "eps must be finite and >= 0");
  for (const float* g : {q_gamma, k_gamma})
    if (!aligned16(g)) return fail(SOL_ERR_INVALID_ARG, "q_gamma and k_gamma must be 16-byte aligned");
  if (k_gamma && !Hk) return fail(SOL_ERR_INVALID_ARG, "k_gamma without k");
  if (dt < 0 || dh < 0 || dw < 0 || dt % 8 || dh % 8 || dw % 8 || (int64_t)dt + dh + dw > D)
    return fail(SOL_ERR_INVALID_ARG, "split must be non-negative multiples of 8, at most %d in all (got %d, %d, %d)", D, dt,
                dh, dw);
  if (T < 0 || Hl < 0 || Wl < 0) return fail(SOL_ERR_INVALID_ARG, "T, Hl, Wl must be >= 0 (got %d, %d, %d)", T, Hl, Wl);
  SOL_TRY(check_small("pos", pos, true));
  SOL_TRY(check_small("lens", lens, true));
  const bool turns = pos && dt + dh + dw > 0;
  if (turns) {
    if (!tab) return fail(SOL_ERR_INVALID_ARG, "rope_tab must not be NULL where there are positions");
    if (!aligned16(tab)) return fail(SOL_ERR_INVALID_ARG, "rope_tab must be 16-byte aligned");
    if (pos_stride_b < 0 || (pos_stride_b && pos_stride_b < 3 * (int64_t)N) || pos_stride_b > kMaxStride)
      return fail(SOL_ERR_INVALID_ARG, "pos_stride_b must be 0 or at least 3 N (got %lld)", (long long)pos_stride_b);
    // a table's pairs are counted in 31 bits, and read from its first plane and its second
    if ((int64_t)T * (dt / 2) + (int64_t)Hl * (dh / 2) + (int64_t)Wl * (dw / 2) > (1 << 28))
      return fail(SOL_ERR_UNSUPPORTED, "T, Hl, Wl too large together (a table of more than 2^28 pairs)");
    s->g = sections(T, Hl, Wl, dt, dh, dw);
  }
  s->B = B;
  s->H = H;
  s->Hk = Hk;
  s->N = N;
  s->eps = eps;
  s->q_gamma = q_gamma;
  s->k_gamma = k_gamma;
  s->pos = turns ? pos : nullptr;
  s->pos_sb = pos_stride_b;
  s->tab = reinterpret_cast<const float2*>(tab);
  s->lens = lens;
  return SOL_OK;
}
// Their spans: in[0 .. 4].
void norm_rope_spans(const sol::NormRope& s, Span* in) {
  in[0] = span("q_gamma", s.q_gamma, sol::kHeadDim * 4);
  in[1] = span("k_gamma", s.k_gamma, sol::kHeadDim * 4);
  in[2] = span("pos", s.pos, ((uint64_t)(s.B - 1) * s.pos_sb + 3 * (uint64_t)s.N) * 4);
  in[3] = span("rope_tab", s.pos ? s.tab : nullptr, (uint64_t)s.g.tab_pairs * 16);
  in[4] = span("lens", s.lens, (uint64_t)s.B * 4);
}
// An output that is its input itself, row for row.
bool in_place(const Span& x, const Span& y) {
  if (!x.bytes || x.at != y.at) return false;
  for (int i = 0; i < 3; ++i)
    if (x.n[i] != y.n[i] || (x.n[i] > 1 && x.s[i] != y.s[i])) return false;
  return true;
}
// Outputs (rows, then the rest) apart from each other and from every input but the
// one that each may be, at the same index.
int check_pairs(const Span* in, int n_in, const Span* out, int n_out, int pairs) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (meet(out[i], in[j]) && !(i == j && i < pairs && in_place(out[i], in[j])))
        return fail(SOL_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, in[j].name);
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return fail(SOL_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, out[j].name);
  }
  return SOL_OK;
}

int check_cross(const sol::CrossShape& s, int D) {
  if (s.B < 1 || s.H < 1 || s.Hk < 1 || s.N < 1 || s.M < 1)
    return fail(SOL_ERR_INVALID_ARG, "B, H, Hk, N, M must be >= 1 (got %d, %d, %d, %d, %d)", s.B, s.H, s.Hk, s.N, s.M);
  if (s.H % s.Hk) return fail(SOL_ERR_INVALID_ARG, "H = %d is not a multiple of Hk = %d", s.H, s.Hk);
  if (D != sol::kHeadDim) return fail(SOL_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", D);
  if (s.N > SOL_MAX_TOKENS || s.M > SOL_MAX_TOKENS)
    return fail(SOL_ERR_UNSUPPORTED, "N=%d or M=%d exceeds %d", s.N, s.M, SOL_MAX_TOKENS);
  // rows and keys are counted in 31 bits
  if ((int64_t)s.B * s.H > (1 << 22) || (int64_t)s.B * s.H * s.N > INT32_MAX || (int64_t)s.B * s.Hk * s.M > INT32_MAX)
    return fail(SOL_ERR_UNSUPPORTED, "B*H, B*H*N or B*Hk*M too large");
  return SOL_OK;
}
int check_cross_call(const sol::CrossShape& s, int D) {
  SOL_TRY(check_cross(s, D));
  if (!std::isfinite(s.scale) || !(s.scale > 0.0f)) return fail(SOL_ERR_INVALID_ARG, "scale must be finite and > 0");
  // a row's log sum over the scale and the lowest maximum, -1e30, times it stay in fp32
  if (s.scale < 1e-30f || s.scale > 1e8f) return fail(SOL_ERR_INVALID_ARG, "scale must be 1e-30 to 1e8 (got %g)", s.scale);
  SOL_TRY(check_small("q_lens", s.q_lens, true));
  SOL_TRY(check_small("kv_lens", s.kv_lens, true));
  return SOL_OK;
}
int check_size(size_t need) {
  if (need == sol::kTooLarge)
    return fail(SOL_ERR_UNSUPPORTED, "B, H, N, M too large together (more than 2^20 tiles of 256 rows, or a launch of 2^32 threads)");
  return SOL_OK;
}
// Their spans: in[0 .. 2].
void cross_spans(const sol::CrossShape& s, Span* in) {
  in[0] = span("q_lens", s.q_lens, (uint64_t)s.B * 4);
  in[1] = span("kv_lens", s.kv_lens, (uint64_t)s.B * 4);
  in[2] = span("key_mask", s.mask, (uint64_t)s.B * s.M);
}
// A shape whose mask is only there or not.
sol::CrossShape cross_shape(int B, int H, int Hk, int N, int M, int masked) {
  static const uint8_t some = 1;
  return {B, H, Hk, N, M, 1.0f, nullptr, nullptr, masked ? &some : nullptr};
}

}  // namespace

extern "C" {

int sol_qk_norm_rope(const void* q, const sol_strides* q_strides, const void* k, const sol_strides* k_strides, void* q_out,
                     const sol_strides* q_out_strides, void* k_out, const sol_strides* k_out_strides, const float* q_gamma,
                     const float* k_gamma, float eps, const int32_t* pos, int64_t pos_stride_b, const float* rope_tab, int T,
                     int Hl, int Wl, int dt, int dh, int dw, const int32_t* lens, int B, int H, int Hk, int N, int D,
                     sol_stream_t stream) {
  sol::NormRopeFwd a = {};
  SOL_TRY(take_norm_rope(&a.s, q_gamma, k_gamma, eps, pos, pos_stride_b, rope_tab, T, Hl, Wl, dt, dh, dw, lens, B, H, Hk, N, D));
  Span in[7] = {}, outs[2] = {};
  SOL_TRY(take_rows("q", q, q_strides, B, H, N, false, &a.q, &in[0]));
  SOL_TRY(take_rows("q_out", q_out, q_out_strides, B, H, N, true, &a.q_out, &outs[0]));
  if (Hk) {
    SOL_TRY(take_rows("k", k, k_strides, B, Hk, N, false, &a.k, &in[1]));
    SOL_TRY(take_rows("k_out", k_out, k_out_strides, B, Hk, N, true, &a.k_out, &outs[1]));
  }
  norm_rope_spans(a.s, in + 2);
  SOL_TRY(check_pairs(in, 7, outs, 2, 2));
  return done(sol::launch_norm_rope_fwd(a, reinterpret_cast<hipStream_t>(stream)), "qk_norm_rope");
}

size_t sol_qk_norm_rope_bwd_workspace_bytes(int B, int H, int Hk, int N, int D) {
  if (check_norm_rope_sizes(B, H, Hk, N, D) != SOL_OK) return 0;
  return sol::norm_rope_bwd_bytes((int64_t)B * N, H + Hk);
}

int sol_qk_norm_rope_bwd(const void* dq_out, const sol_strides* dq_out_strides, const void* dk_out,
                         const sol_strides* dk_out_strides, const void* q, const sol_strides* q_strides, const void* k,
                         const sol_strides* k_strides, void* dq, const sol_strides* dq_strides, void* dk,
                         const sol_strides* dk_strides, const float* q_gamma, const float* k_gamma, float* dq_gamma,
                         float* dk_gamma, float eps, const int32_t* pos, int64_t pos_stride_b, const float* rope_tab, int T,
                         int Hl, int Wl, int dt, int dh, int dw, const int32_t* lens, int B, int H, int Hk, int N, int D,
                         void* workspace, size_t workspace_bytes, sol_stream_t stream) {
  sol::NormRopeBwd a = {};
  SOL_TRY(take_norm_rope(&a.s, q_gamma, k_gamma, eps, pos, pos_stride_b, rope_tab, T, Hl, Wl, dt, dh, dw, lens, B, H, Hk, N, D));
  Span in[9] = {}, outs[5] = {};
  SOL_TRY(take_rows("dq_out", dq_out, dq_out_strides, B, H, N, false, &a.dq_out, &in[0]));
  SOL_TRY(take_rows("dq", dq, dq_strides, B, H, N, true, &a.dq, &outs[0]));
  // (without a norm the gradients do not ask what q and k were)
  if (q_gamma) SOL_TRY(take_rows("q", q, q_strides, B, H, N, false, &a.q, &in[2]));
  if (Hk) {
    SOL_TRY(take_rows("dk_out", dk_out, dk_out_strides, B, Hk, N, false, &a.dk_out, &in[1]));
    SOL_TRY(take_rows("dk", dk, dk_strides, B, Hk, N, true, &a.dk, &outs[1]));
    if (k_gamma) SOL_TRY(take_rows("k", k, k_strides, B, Hk, N, false, &a.k, &in[3]));
  }
  if ((dq_gamma && !q_gamma) || (dk_gamma && !k_gamma))
    return fail(SOL_ERR_INVALID_ARG, "a gradient of weights that are not there (dq_gamma, dk_gamma)");
  SOL_TRY(check_small("dq_gamma", dq_gamma, true));
  SOL_TRY(check_small("dk_gamma", dk_gamma, true));
  const size_t need = dq_gamma || dk_gamma ? sol::norm_rope_bwd_bytes((int64_t)B * N, H + Hk) : 0;
  SOL_TRY(check_workspace(workspace, workspace_bytes, need));
  norm_rope_spans(a.s, in + 4);
  outs[2] = span("dq_gamma", dq_gamma, sol::kHeadDim * 4);
  outs[3] = span("dk_gamma", dk_gamma, sol::kHeadDim * 4);
  outs[4] = span("workspace", workspace, need);
  SOL_TRY(check_pairs(in, 9, outs, 5, 2));
  a.dq_gamma = dq_gamma;
  a.dk_gamma = dk_gamma;
  a.partial = need ? static_cast<float*>(workspace) : nullptr;
  return done(sol::launch_norm_rope_bwd(a, reinterpret_cast<hipStream_t>(stream)), "qk_norm_rope_bwd");
}

size_t sol_cross_attn_fwd_workspace_bytes(int B, int H, int Hk, int N, int M, int D, int masked) {
  const sol::CrossShape s = cross_shape(B, H, Hk, N, M, masked);
  if (check_cross(s, D) != SOL_OK) return 0;
  const size_t need = sol::cross_fwd_bytes(s, nullptr, nullptr);
  return check_size(need) == SOL_OK ? need : 0;
}

size_t sol_cross_attn_bwd_workspace_bytes(int B, int H, int Hk, int N, int M, int D, int masked) {
  const sol::CrossShape s = cross_shape(B, H, Hk, N, M, masked);
  if (check_cross(s, D) != SOL_OK) return 0;
  const size_t need = sol::cross_bwd_bytes(s, nullptr, nullptr);
  return check_size(need) == SOL_OK ? need : 0;
}

int sol_cross_attn_fwd(const void* q, const sol_strides* q_strides, const void* k, const sol_strides* k_strides,
                       const void* v, const sol_strides* v_strides, void* out, const sol_strides* out_strides,
                       void* out_left, float* lse, const int32_t* q_lens, const int32_t* kv_lens, const uint8_t* key_mask,
                       int B, int H, int Hk, int N, int M, int D, float scale, void* workspace, size_t workspace_bytes,
                       sol_stream_t stream) {
  sol::CrossFwd a = {};
  a.s = {B, H, Hk, N, M, scale, q_lens, kv_lens, key_mask};
  SOL_TRY(check_cross_call(a.s, D));
  Span in[6], outs[4];
  SOL_TRY(take_rows("q", q, q_strides, B, H, N, false, &a.q, &in[0]));
  SOL_TRY(take_rows("k", k, k_strides, B, Hk, M, false, &a.k, &in[1]));
  SOL_TRY(take_rows("v", v, v_strides, B, Hk, M, false, &a.v, &in[2]));
  SOL_TRY(take_rows("out", out, out_strides, B, H, N, true, &a.out, &outs[0]));
  if (!aligned16(out_left)) return fail(SOL_ERR_INVALID_ARG, "out_left must be 16-byte aligned");
  SOL_TRY(check_small("lse", lse, true));
  if (!out_left != !lse) return fail(SOL_ERR_INVALID_ARG, "out_left and lse are given together or not at all");
  const size_t need = sol::cross_fwd_bytes(a.s, &a, workspace);
  SOL_TRY(check_size(need));
  SOL_TRY(check_workspace(workspace, workspace_bytes, need));
  cross_spans(a.s, in + 3);
  outs[1] = span("out_left", out_left, (uint64_t)B * H * N * D * 2);
  outs[2] = span("lse", lse, (uint64_t)B * H * N * 4);
  outs[3] = span("workspace", workspace, need);
  SOL_TRY(check_apart(in, 6, outs, 4));
  a.left = static_cast<uint16_t*>(out_left);
  a.lse = lse;
  return done(sol::launch_cross_fwd(a, reinterpret_cast<hipStream_t>(stream)), "cross_attn_fwd");
}

int sol_cross_attn_bwd(const void* dout, const sol_strides* dout_strides, const void* q, const sol_strides* q_strides,
                       const void* k, const sol_strides* k_strides, const void* v, const sol_strides* v_strides,
                       const void* out, const sol_strides* out_strides, const void* out_left, const float* lse, void* dq,
                       const sol_strides* dq_strides, void* dk, const sol_strides* dk_strides, void* dv,
                       const sol_strides* dv_strides, const int32_t* q_lens, const int32_t* kv_lens,
                       const uint8_t* key_mask, int B, int H, int Hk, int N, int M, int D, float scale, void* workspace,
                       size_t workspace_bytes, sol_stream_t stream) {
  sol::CrossBwd a = {};
  a.s = {B, H, Hk, N, M, scale, q_lens, kv_lens, key_mask};
  SOL_TRY(check_cross_call(a.s, D));
  Span in[10], outs[4];
  SOL_TRY(take_rows("dout", dout, dout_strides, B, H, N, false, &a.dout, &in[0]));
  SOL_TRY(take_rows("q", q, q_strides, B, H, N, false, &a.q, &in[1]));
  SOL_TRY(take_rows("k", k, k_strides, B, Hk, M, false, &a.k, &in[2]));
  SOL_TRY(take_rows("v", v, v_strides, B, Hk, M, false, &a.v, &in[3]));
  SOL_TRY(take_rows("out", out, out_strides, B, H, N, false, &a.out, &in[4]));
  SOL_TRY(take_rows("dq", dq, dq_strides, B, H, N, true, &a.dq, &outs[0]));
  SOL_TRY(take_rows("dk", dk, dk_strides, B, Hk, M, true, &a.dk, &outs[1]));
  SOL_TRY(take_rows("dv", dv, dv_strides, B, Hk, M, true, &a.dv, &outs[2]));
  if (!out_left) return fail(SOL_ERR_INVALID_ARG, "out_left must not be NULL");
  if (!aligned16(out_left)) return fail(SOL_ERR_INVALID_ARG, "out_left must be 16-byte aligned");
  SOL_TRY(check_small("lse", lse, false));
  const size_t need = sol::cross_bwd_bytes(a.s, &a, workspace);
  SOL_TRY(check_size(need));
  SOL_TRY(check_workspace(workspace, workspace_bytes, need));
  in[5] = span("out_left", out_left, (uint64_t)B * H * N * D * 2);
  in[6] = span("lse", lse, (uint64_t)B * H * N * 4);
  cross_spans(a.s, in + 7);
  outs[3] = span("workspace", workspace, need);
  SOL_TRY(check_apart(in, 10, outs, 4));
  a.left = static_cast<const uint16_t*>(out_left);
  a.lse = lse;
  return done(sol::launch_cross_bwd(a, reinterpret_cast<hipStream_t>(stream)), "cross_attn_bwd");
}

}  // extern "C"
