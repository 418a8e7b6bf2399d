// C ABI front end of the linear and differential attention: argument
// validation (before any HIP call), launch and error mapping.
#include <cmath>

#include "sol_checks.h"
#include "sol_ops.h"

namespace {

// (b, h) slabs of a linear call.  A launch is a 1D grid of fewer than 2^32
// threads: three scans of 512 a slab, or four workgroups of 256 a request and
// head; segments add to a call of few slabs only.
constexpr int64_t kMaxSlabs = (int64_t)1 << 21;
int check_slabs(const char* what, int64_t slabs) {
  if (slabs > kMaxSlabs) return fail(SOL_ERR_UNSUPPORTED, "%s too large (at most 2^21)", what);
  return SOL_OK;
}

// The sum of shared heads' gradients runs one thread per 16-byte chunk of dk and dv.
int check_group_sum(int B, int H, int Hk, int N) {
  if (Hk < H && (int64_t)B * Hk * N > ((int64_t)1 << 26)) return fail(SOL_ERR_UNSUPPORTED, "B*Hk*N too large");
  return SOL_OK;
}

// The sizes of a differential call.
int check_diff_sizes(const sol::DiffShape& s, int D) {
  if (s.B < 1 || s.H < 1 || s.Hv < 1 || s.N < 1 || s.M < 1)
    return fail(SOL_ERR_INVALID_ARG, "B, H, Hv, N, M must be >= 1 (got %d, %d, %d, %d, %d)", s.B, s.H, s.Hv, s.N, s.M);
  if (s.H % s.Hv) return fail(SOL_ERR_INVALID_ARG, "H = %d is not a multiple of Hv = %d", s.H, s.Hv);
  if (s.Hk != s.Hv && s.Hk != 2 * (int64_t)s.Hv)
    return fail(SOL_ERR_INVALID_ARG, "Hk must be Hv or 2 Hv (got %d for Hv = %d)", s.Hk, s.Hv);
  if (D != sol::kHeadDim) return fail(SOL_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", D);
  if (s.N > SOL_MAX_TOKENS || s.M > SOL_MAX_TOKENS)
    return fail(SOL_ERR_UNSUPPORTED, "N=%d or M=%d exceeds %d", s.N, s.M, SOL_MAX_TOKENS);
  // rows and keys are counted in 31 bits
  if ((int64_t)s.B * s.H > (1 << 22) || (int64_t)s.B * s.H * s.N > INT32_MAX || (int64_t)s.B * s.Hv * s.M > INT32_MAX)
    return fail(SOL_ERR_UNSUPPORTED, "B*H, B*H*N or B*Hv*M too large");
  return SOL_OK;
}
int check_launch(size_t need) {
  if (need == sol::kTooLarge)
    return fail(SOL_ERR_UNSUPPORTED, "B, H, N, M too large together (a launch of 2^32 threads or more)");
  return SOL_OK;
}
int check_diff(const sol::DiffShape& s, int D) {
  SOL_TRY(check_diff_sizes(s, D));
  if (!std::isfinite(s.scale) || !(s.scale > 0.0f)) return fail(SOL_ERR_INVALID_ARG, "scale must be finite and > 0");
  // a row's log sum over the scale and the lowest maximum, -1e30, times it stay in fp32
  if (s.scale < 1e-30f || s.scale > 1e8f) return fail(SOL_ERR_INVALID_ARG, "scale must be 1e-30 to 1e8 (got %g)", s.scale);
  SOL_TRY(check_small("lambda", s.lambda, false));
  SOL_TRY(check_small("q_lens", s.q_lens, true));
  SOL_TRY(check_small("kv_lens", s.kv_lens, true));
  return SOL_OK;
}

constexpr uint64_t kStateBytes = (uint64_t)sol::kStateElems * sizeof(float);

}  // namespace

extern "C" {

size_t sol_lin_attn_fwd_workspace_bytes(int B, int H, int N, int D) {
  if (check_heads(B, H, H, N, D) != SOL_OK || check_slabs("B*H", (int64_t)B * H) != SOL_OK) return 0;
  return sol::lin_states_bytes((int64_t)B * H, N, 1);
}

size_t sol_lin_attn_bwd_workspace_bytes(int B, int H, int Hk, int N, int D) {
  if (check_heads(B, H, Hk, N, D) != SOL_OK || check_slabs("B*H", (int64_t)B * H) != SOL_OK ||
      check_group_sum(B, H, Hk, N) != SOL_OK)
    return 0;
  const size_t partial = Hk < H ? (size_t)2 * B * H * N * D * sizeof(float) : 0;
  return up256(sol::lin_states_bytes((int64_t)B * H, N, 3)) + partial;
}

int sol_lin_attn_fwd(const void* q, const sol_strides* q_strides, const void* k, const sol_strides* k_strides,
                     const void* v, const sol_strides* v_strides, void* out, const sol_strides* out_strides,
                     const float* log_decay, const float* state_in, float* state_out, const int32_t* lens, int B, int H,
                     int Hk, int N, int D, float scale, void* workspace, size_t workspace_bytes, sol_stream_t stream) {
  SOL_TRY(check_heads(B, H, Hk, N, D));
  SOL_TRY(check_slabs("B*H", (int64_t)B * H));
  sol::LinFwd a = {};
  Span in[6], outs[3];
  SOL_TRY(take_rows("q", q, q_strides, B, H, N, false, &a.q, &in[0]));
  SOL_TRY(take_rows("k", k, k_strides, B, Hk, N, false, &a.k, &in[1]));
  SOL_TRY(take_rows("v", v, v_strides, B, Hk, N, false, &a.v, &in[2]));
  SOL_TRY(take_rows("out", out, out_strides, B, H, N, true, &a.out, &outs[0]));
  SOL_TRY(check_small("log_decay", log_decay, false));
  SOL_TRY(check_small("lens", lens, true));
  if (!aligned16(state_in) || !aligned16(state_out))
    return fail(SOL_ERR_INVALID_ARG, "state_in and state_out must be 16-byte aligned");
  if (!std::isfinite(scale)) return fail(SOL_ERR_INVALID_ARG, "scale must be finite");
  const size_t need = sol_lin_attn_fwd_workspace_bytes(B, H, N, D);
  SOL_TRY(check_workspace(workspace, workspace_bytes, need));
  const uint64_t states = (uint64_t)B * H * kStateBytes;
  in[3] = span("log_decay", log_decay, (uint64_t)H * 4);
  in[4] = span("lens", lens, (uint64_t)B * 4);
  in[5] = span("state_in", state_out == state_in ? nullptr : state_in, states);
  outs[1] = span("state_out", state_out, states);
  outs[2] = span("workspace", workspace, need);
  SOL_TRY(check_apart(in, 6, outs, 3));
  if (state_out == state_in && state_in) {
    // in place: the state is an input of this call all the same
    const Span s = span("state_in", state_in, states);
    if (meet(outs[0], s) || meet(outs[2], s)) return fail(SOL_ERR_INVALID_ARG, "state_in overlaps out or workspace");
  }
  a.log_decay = log_decay;
  a.state_in = state_in;
  a.state_out = state_out;
  a.lens = lens;
  a.B = B;
  a.H = H;
  a.Hk = Hk;
  a.N = N;
  a.scale = scale;
  a.states = static_cast<float*>(workspace);
  return done(sol::launch_lin_fwd(a, reinterpret_cast<hipStream_t>(stream)), "lin_attn_fwd");
}

int sol_lin_attn_bwd(const void* dout, const sol_strides* dout_strides, const void* q, const sol_strides* q_strides,
                     const void* k, const sol_strides* k_strides, const void* v, const sol_strides* v_strides, void* dq,
                     const sol_strides* dq_strides, void* dk, const sol_strides* dk_strides, void* dv,
                     const sol_strides* dv_strides, const float* log_decay, const float* state_in,
                     const float* dstate_out, float* dstate_in, const int32_t* lens, int B, int H, int Hk, int N, int D,
                     float scale, void* workspace, size_t workspace_bytes, sol_stream_t stream) {
  SOL_TRY(check_heads(B, H, Hk, N, D));
  SOL_TRY(check_slabs("B*H", (int64_t)B * H));
  SOL_TRY(check_group_sum(B, H, Hk, N));
  sol::LinBwd a = {};
  Span in[8], outs[5];
  SOL_TRY(take_rows("dout", dout, dout_strides, B, H, N, false, &a.dout, &in[0]));
  SOL_TRY(take_rows("q", q, q_strides, B, H, N, false, &a.q, &in[1]));
  SOL_TRY(take_rows("k", k, k_strides, B, Hk, N, false, &a.k, &in[2]));
  SOL_TRY(take_rows("v", v, v_strides, B, Hk, N, false, &a.v, &in[3]));
  SOL_TRY(take_rows("dq", dq, dq_strides, B, H, N, true, &a.dq, &outs[0]));
  SOL_TRY(take_rows("dk", dk, dk_strides, B, Hk, N, true, &a.dk, &outs[1]));
  SOL_TRY(take_rows("dv", dv, dv_strides, B, Hk, N, true, &a.dv, &outs[2]));
  SOL_TRY(check_small("log_decay", log_decay, false));
  SOL_TRY(check_small("lens", lens, true));
  if (!aligned16(state_in) || !aligned16(dstate_out) || !aligned16(dstate_in))
    return fail(SOL_ERR_INVALID_ARG, "state_in, dstate_out and dstate_in must be 16-byte aligned");
  if (!std::isfinite(scale)) return fail(SOL_ERR_INVALID_ARG, "scale must be finite");
  const size_t need = sol_lin_attn_bwd_workspace_bytes(B, H, Hk, N, D);
  SOL_TRY(check_workspace(workspace, workspace_bytes, need));
  const uint64_t states = (uint64_t)B * H * kStateBytes;
  const bool in_place = dstate_in && dstate_in == dstate_out;
  in[4] = span("log_decay", log_decay, (uint64_t)H * 4);
  in[5] = span("lens", lens, (uint64_t)B * 4);
  in[6] = span("state_in", state_in, states);
  in[7] = span("dstate_out", in_place ? nullptr : dstate_out, states);
  outs[3] = span("dstate_in", dstate_in, states);
  outs[4] = span("workspace", workspace, need);
  SOL_TRY(check_apart(in, 8, outs, 5));
  a.log_decay = log_decay;
  a.state_in = state_in;
  a.dstate_in = dstate_out;
  a.dstate_out = dstate_in;
  a.lens = lens;
  a.B = B;
  a.H = H;
  a.Hk = Hk;
  a.N = N;
  a.scale = scale;
  a.states = static_cast<float*>(workspace);
  if (Hk < H)
    a.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                         up256(sol::lin_states_bytes((int64_t)B * H, N, 3)));
  return done(sol::launch_lin_bwd(a, reinterpret_cast<hipStream_t>(stream)), "lin_attn_bwd");
}

int sol_lin_attn_step(const void* q, const sol_strides* q_strides, const void* k, const sol_strides* k_strides,
                      const void* v, const sol_strides* v_strides, void* out, const sol_strides* out_strides,
                      const float* log_decay, float* state, const int32_t* slots, int R, int H, int Hk, int n_slots,
                      int D, float scale, sol_stream_t stream) {
  SOL_TRY(check_heads(R, H, Hk, 1, D));
  SOL_TRY(check_slabs("R*H", (int64_t)R * H));
  if (n_slots < 1) return fail(SOL_ERR_INVALID_ARG, "n_slots must be >= 1 (got %d)", n_slots);
  if (!slots && R > n_slots) return fail(SOL_ERR_INVALID_ARG, "%d requests without slots, a pool of %d", R, n_slots);
  sol::LinStep a = {};
  Span in[5], outs[2];
  SOL_TRY(take_rows("q", q, q_strides, R, H, 1, false, &a.q, &in[0]));
  SOL_TRY(take_rows("k", k, k_strides, R, Hk, 1, false, &a.k, &in[1]));
  SOL_TRY(take_rows("v", v, v_strides, R, Hk, 1, false, &a.v, &in[2]));
  SOL_TRY(take_rows("out", out, out_strides, R, H, 1, true, &a.out, &outs[0]));
  SOL_TRY(check_small("log_decay", log_decay, false));
  SOL_TRY(check_small("slots", slots, true));
  if (!state) return fail(SOL_ERR_INVALID_ARG, "state must not be NULL");
  if (!aligned16(state)) return fail(SOL_ERR_INVALID_ARG, "state must be 16-byte aligned");
  if (!std::isfinite(scale)) return fail(SOL_ERR_INVALID_ARG, "scale must be finite");
  in[3] = span("log_decay", log_decay, (uint64_t)H * 4);
  in[4] = span("slots", slots, (uint64_t)R * 4);
  outs[1] = span("state", state, (uint64_t)n_slots * H * kStateBytes);
  SOL_TRY(check_apart(in, 5, outs, 2));
  a.log_decay = log_decay;
  a.state = state;
  a.slots = slots;
  a.R = R;
  a.H = H;
  a.Hk = Hk;
  a.n_slots = n_slots;
  a.scale = scale;
  return done(sol::launch_lin_step(a, reinterpret_cast<hipStream_t>(stream)), "lin_attn_step");
}

size_t sol_diff_attn_fwd_workspace_bytes(int B, int H, int Hv, int N, int M, int D) {
  sol::DiffShape s = {B, H, Hv, Hv, N, M, 1.0f, 0, nullptr, nullptr, nullptr};
  if (check_diff_sizes(s, D) != SOL_OK) return 0;
  // the larger of the two masks'
  const size_t all = sol::diff_fwd_bytes(s);
  s.causal = 1;
  const size_t causal = sol::diff_fwd_bytes(s);
  const size_t most = all > causal ? all : causal;
  return check_launch(most) == SOL_OK ? most : 0;
}

size_t sol_diff_attn_bwd_workspace_bytes(int B, int H, int Hv, int N, int M, int D) {
  sol::DiffShape s = {B, H, Hv, Hv, N, M, 1.0f, 0, nullptr, nullptr, nullptr};
  if (check_diff_sizes(s, D) != SOL_OK) return 0;
  const size_t all = sol::diff_bwd_bytes(s, nullptr);
  s.causal = 1;
  const size_t causal = sol::diff_bwd_bytes(s, nullptr);
  const size_t most = all > causal ? all : causal;
  return check_launch(most) == SOL_OK ? most : 0;
}

int sol_diff_attn_fwd(const void* q, const sol_strides* q_strides, const void* k, const sol_strides* k_strides,
                      const void* v, const sol_strides* v_strides, void* out, const sol_strides* out_strides,
                      void* out2, float* lse, const float* lambda, const int32_t* q_lens, const int32_t* kv_lens, int B,
                      int H, int Hv, int Hk, int N, int M, int D, float scale, int causal, void* workspace,
                      size_t workspace_bytes, sol_stream_t stream) {
  sol::DiffFwd a = {};
  a.s = {B, H, Hv, Hk, N, M, scale, causal != 0, q_lens, kv_lens, lambda};
  SOL_TRY(check_diff(a.s, D));
  Span in[6], outs[4];
  SOL_TRY(take_rows("q", q, q_strides, B, 2 * H, N, false, &a.q, &in[0]));
  SOL_TRY(take_rows("k", k, k_strides, B, Hk, M, false, &a.k, &in[1]));
  SOL_TRY(take_rows("v", v, v_strides, B, Hv, M, false, &a.v, &in[2]));
  SOL_TRY(take_rows("out", out, out_strides, B, H, N, true, &a.out, &outs[0]));
  if (!aligned16(out2)) return fail(SOL_ERR_INVALID_ARG, "out2 must be 16-byte aligned");
  SOL_TRY(check_small("lse", lse, true));
  if (!out2 != !lse) return fail(SOL_ERR_INVALID_ARG, "out2 and lse are given together or not at all");
  const size_t need = sol::diff_fwd_bytes(a.s);
  SOL_TRY(check_launch(need));
  SOL_TRY(check_workspace(workspace, workspace_bytes, need));
  in[3] = span("lambda", lambda, (uint64_t)H * 4);
  in[4] = span("q_lens", q_lens, (uint64_t)B * 4);
  in[5] = span("kv_lens", kv_lens, (uint64_t)B * 4);
  outs[1] = span("out2", out2, (uint64_t)B * H * N * D * 6);
  outs[2] = span("lse", lse, (uint64_t)B * 2 * H * N * 4);
  outs[3] = span("workspace", workspace, need);
  SOL_TRY(check_apart(in, 6, outs, 4));
  a.out2 = static_cast<uint16_t*>(out2);
  a.lse = lse;
  a.ws = static_cast<float*>(workspace);
  return done(sol::launch_diff_fwd(a, reinterpret_cast<hipStream_t>(stream)), "diff_attn_fwd");
}

int sol_diff_attn_bwd(const void* dout, const sol_strides* dout_strides, const void* q, const sol_strides* q_strides,
                      const void* k, const sol_strides* k_strides, const void* v, const sol_strides* v_strides,
                      const void* out, const sol_strides* out_strides, const void* out2, const float* lse,
                      const float* lambda, void* dq, const sol_strides* dq_strides, void* dk,
                      const sol_strides* dk_strides, void* dv, const sol_strides* dv_strides, float* dlambda,
                      const int32_t* q_lens, const int32_t* kv_lens, int B, int H, int Hv, int Hk, int N, int M, int D,
                      float scale, int causal, void* workspace, size_t workspace_bytes, sol_stream_t stream) {
  sol::DiffBwd a = {};
  a.s = {B, H, Hv, Hk, N, M, scale, causal != 0, q_lens, kv_lens, lambda};
  SOL_TRY(check_diff(a.s, D));
  Span in[10], outs[5];
  SOL_TRY(take_rows("dout", dout, dout_strides, B, H, N, false, &a.dout, &in[0]));
  SOL_TRY(take_rows("q", q, q_strides, B, 2 * H, N, false, &a.q, &in[1]));
  SOL_TRY(take_rows("k", k, k_strides, B, Hk, M, false, &a.k, &in[2]));
  SOL_TRY(take_rows("v", v, v_strides, B, Hv, M, false, &a.v, &in[3]));
  SOL_TRY(take_rows("out", out, out_strides, B, H, N, false, &a.out, &in[4]));
  SOL_TRY(take_rows("dq", dq, dq_strides, B, 2 * H, N, true, &a.dq, &outs[0]));
  SOL_TRY(take_rows("dk", dk, dk_strides, B, Hk, M, true, &a.dk, &outs[1]));
  SOL_TRY(take_rows("dv", dv, dv_strides, B, Hv, M, true, &a.dv, &outs[2]));
  if (!out2) return fail(SOL_ERR_INVALID_ARG, "out2 must not be NULL");
  if (!aligned16(out2)) return fail(SOL_ERR_INVALID_ARG, "out2 must be 16-byte aligned");
  SOL_TRY(check_small("lse", lse, false));
  SOL_TRY(check_small("dlambda", dlambda, false));
  a.stats = static_cast<float*>(workspace);
  const size_t need = sol::diff_bwd_bytes(a.s, &a);
  SOL_TRY(check_launch(need));
  SOL_TRY(check_workspace(workspace, workspace_bytes, need));
  in[5] = span("out2", out2, (uint64_t)B * H * N * D * 6);
  in[6] = span("lse", lse, (uint64_t)B * 2 * H * N * 4);
  in[7] = span("lambda", lambda, (uint64_t)H * 4);
  in[8] = span("q_lens", q_lens, (uint64_t)B * 4);
  in[9] = span("kv_lens", kv_lens, (uint64_t)B * 4);
  outs[3] = span("dlambda", dlambda, (uint64_t)H * 4);
  outs[4] = span("workspace", workspace, need);
  SOL_TRY(check_apart(in, 10, outs, 5));
  a.out2 = static_cast<const uint16_t*>(out2);
  a.lse = lse;
  a.dlambda = dlambda;
  return done(sol::launch_diff_bwd(a, reinterpret_cast<hipStream_t>(stream)), "diff_attn_bwd");
}

}  // extern "C"
