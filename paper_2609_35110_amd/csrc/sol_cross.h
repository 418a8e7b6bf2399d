// Internal interface of the norm and rotation at positions of their own
// (sol_qk_norm_rope*) and of cross attention (sol_cross_attn_*): what the front
// end (sol_api_cross.cpp) hands the HIP launchers (sol_norm_rope.hip,
// sol_cross_attn.hip).  Arguments reaching the launchers have been validated
// already.
#pragma once

#include "sol_ops.h"

namespace sol {

// ------------------------------------- norm and rotation at given positions

// What both directions share.  Hk is 0 where there is no k.
struct NormRope {
  int B, H, Hk, N;
  float eps;
  const float *q_gamma, *k_gamma;  // may be null (no norm)
  const int32_t* pos;              // [3] of token (b, n) at b pos_sb + 3 n; null: nothing rotates
  int64_t pos_sb;
  const float2* tab;  // of an extent T x Hl x Wl and the split
  SeqGrid g;          // the table's sections (n, nt, hw unused)
  const int32_t* lens;  // may be null (all N)
};

struct NormRopeFwd {
  NormRope s;
  Rows q, k, q_out, k_out;
};
hipError_t launch_norm_rope_fwd(const NormRopeFwd& a, hipStream_t stream);

struct NormRopeBwd {
  NormRope s;
  Rows dq_out, dk_out, q, k, dq, dk;
  float *dq_gamma, *dk_gamma;  // null: no norm, or not wanted
  float* partial;              // fp32 [workgroup][2][128], where a gamma's gradient is wanted
};
// Bytes of workspace where a gamma's gradient is wanted (heads: of q and k).
size_t norm_rope_bwd_bytes(int64_t tokens, int heads);
hipError_t launch_norm_rope_bwd(const NormRopeBwd& a, hipStream_t stream);

// ------------------------------------------------------------ cross attention

constexpr int kCrossRows = 256;  // query rows of a workgroup of the tile kernels
constexpr int kCrossKeys = 128;  // keys of a workgroup of dk and dv's kernel

struct CrossShape {
  int B, H, Hk, N, M;
  float scale;
  const int32_t* q_lens;   // may be null (all N)
  const int32_t* kv_lens;  // may be null (all M)
  const uint8_t* mask;     // [B][M], 0: hidden; may be null
};

// How a forward call runs: in groups of few rows that share a key head, their keys in
// `pieces` (few); or in tiles of rows that workgroups take in line, all of a head's keys in
// LDS (brief), or a ring of them, tiles shared at the workgroups' borders (split) or not.
constexpr int kShortKeys = 256;
struct CrossPlan {
  bool few;
  int pieces;
  bool brief;
  bool split;
  int workgroups;  // of the tile kernel
};
constexpr int kCus = 256;  // compute units: each holds one workgroup of the tile kernels
CrossPlan cross_plan(const CrossShape& s, bool ragged);  // ragged: with q_lens, kv_lens or mask

struct CrossFwd {
  CrossShape s;
  Rows q, k, v, out;
  // For the gradients (both null or neither): what out's rounding left, bf16
  // [B][H][N][128]; the rows' log sums, [B][H][N].
  uint16_t* left;
  float* lse;
  float* ws;
  // Where keys are masked and the tile kernels run: [B][M], the visible keys of a
  // sequence in order and then the others; [B], how many are visible.
  int32_t *order, *counts;
};
// Bytes of workspace, with lengths or without (or kTooLarge); with a given, its sections
// (from ws on) are filled in.
size_t cross_fwd_bytes(const CrossShape& s, CrossFwd* a, void* ws);
hipError_t launch_cross_fwd(const CrossFwd& a, hipStream_t stream);

struct CrossBwd {
  CrossShape s;
  Rows q, k, v, out, dout, dq, dk, dv;
  const uint16_t* left;
  const float* lse;
  int32_t *order, *counts;  // as above
  float* stats;      // [B][H][ceil(N / 32)][2][32]
  float* dq_parts;   // [row tile that is cut][piece][256][128]
  float* dkv_parts;  // [key tile][piece][dv, dk][128][128], several pieces
  DiffTiles plan;
  // A key tile's query heads and their rows in head_pieces x row_pieces workgroups
  // (head_pieces divides H / Hk, and is that where row_pieces > 1).
  int head_pieces, row_pieces;
};
// Bytes of workspace, or kTooLarge; with a given, its sections (from ws on) and plan
// are filled in.
size_t cross_bwd_bytes(const CrossShape& s, CrossBwd* a, void* ws);
hipError_t launch_cross_bwd(const CrossBwd& a, hipStream_t stream);

}  // namespace sol
