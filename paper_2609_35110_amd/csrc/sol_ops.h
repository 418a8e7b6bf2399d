// Internal interface of the linear (sol_lin_attn_*) and differential
// (sol_diff_attn_*) attention: what the front end (sol_api_ops.cpp) hands the
// HIP launchers (sol_lin_attn.hip, sol_diff_attn.hip).  Arguments reaching the
// launchers have been validated already.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sol.h"
#include "sol_internal.h"

namespace sol {

// Rows of 128 bf16: row (b, h, n) at element b sb + h sh + n sn of p.
struct Rows {
  uint16_t* p;
  int64_t sb, sh, sn;
};

// ------------------------------------------------- linear attention, decayed

constexpr int kLinRows = 64;                      // tokens per chunk of the scan
constexpr int kStateElems = kHeadDim * kHeadDim;  // fp32 values of a head's state

// Tokens of a sequence that one workgroup walks, and the segments that makes:
// the scan is sequential in the tokens, so a call of few (b, h) slabs splits
// its tokens into segments whose states are found first (one pass over k and v
// and one over the segments' states).
struct LinPlan {
  int seg_rows;  // a multiple of kLinRows
  int nseg;
  int parts;  // of a segment, in the pass that finds its state (divide its chunks)
};
LinPlan lin_plan(int64_t slabs, int N, int scans);
// Bytes of the segments' states (0 for one segment).
size_t lin_states_bytes(int64_t slabs, int N, int scans);

// out = scale (scan of q, k, v), state_out = the final state (fp32, may be
// null or state_in itself); states: lin_states_bytes of workspace.
struct LinFwd {
  Rows q, k, v, out;
  const float* log_decay;
  const float* state_in;  // may be null (zero)
  float* state_out;
  const int32_t* lens;  // may be null (all N)
  int B, H, Hk, N;
  float scale;
  float* states;
};
hipError_t launch_lin_fwd(const LinFwd& a, hipStream_t stream);

struct LinBwd {
  Rows q, k, v, dout, dq, dk, dv;
  const float* log_decay;
  const float* state_in;   // may be null
  const float* dstate_in;  // gradient of the final state, may be null
  float* dstate_out;       // gradient of the initial state, may be null
  const int32_t* lens;
  int B, H, Hk, N;
  float scale;
  float* states;
  float* partial;  // fp32 [2][B][H][N][128] when Hk < H, else null
};
hipError_t launch_lin_bwd(const LinBwd& a, hipStream_t stream);

struct LinStep {
  Rows q, k, v, out;  // sn unused
  const float* log_decay;
  float* state;  // fp32 [n_slots][H][128][128]
  const int32_t* slots;  // may be null (request r has slot r)
  int R, H, Hk, n_slots;
  float scale;
};
hipError_t launch_lin_step(const LinStep& a, hipStream_t stream);

// ------------------------------------------------------ differential attention

constexpr int kDiffRows = 128;  // query rows of a workgroup
constexpr int kDiffKeys = 64;   // keys of a tile
constexpr int kFewRows = 32;    // (head of a group, token) rows of the few-row kernel

// In place of a call's workspace: its launches would have 2^32 threads or more.
constexpr size_t kTooLarge = ~(size_t)0;

// What both directions share.  Hk is Hv (both maps read one key head) or 2 Hv.
struct DiffShape {
  int B, H, Hv, Hk, N, M;
  float scale;
  int causal;
  const int32_t* q_lens;   // may be null
  const int32_t* kv_lens;  // may be null
  const float* lambda;
};

// Row tiles [0, full) whole, the others in `pieces` pieces of their keys, whose
// results another launch joins through the workspace.
struct DiffTiles {
  int full, pieces;
};
// How a forward call runs: with so few rows that a group's fit one wave (few,
// its workgroups all cut), or in row tiles.
struct DiffPlan {
  bool few;
  DiffTiles tiles;
};
DiffPlan diff_plan(const DiffShape& s, bool ragged);  // ragged: with kv_lens
size_t diff_fwd_bytes(const DiffShape& s);  // (or kTooLarge)

struct DiffFwd {
  DiffShape s;
  Rows q, k, v, out;
  // For the gradients (both null or neither): [B][H][N][3][128], the second map's
  // own output, what its rounding left, and what that of out left; [B][2H][N].
  uint16_t* out2;
  float* lse;
  float* ws;
};
hipError_t launch_diff_fwd(const DiffFwd& a, hipStream_t stream);

struct DiffBwd {
  DiffShape s;
  Rows q, k, v, out, dout, dq, dk, dv;
  const uint16_t* out2;
  const float* lse;
  float* dlambda;
  float* stats;    // [B][H][ceil(N / 32)][4][32]: the workspace's start
  float* delta;    // [B][H][ceil(N / 32)]
  float* partial;  // [H][B][parts], parts 4 a key tile and row piece
  float* dq_parts; // [row tile that is cut][piece][map][128][128]
  int parts;
  DiffTiles plan;
  // A key tile's query heads and their rows in head_pieces x row_pieces workgroups
  // (head_pieces divides H / Hv, and is that where row_pieces > 1).
  int head_pieces, row_pieces;
  float* dkv_parts;  // [key tile][piece][dv, dk of each map][128][128], several pieces
};
// Bytes of workspace, or kTooLarge; with a given, its sections and plan are filled
// in (from a->stats on).
size_t diff_bwd_bytes(const DiffShape& s, DiffBwd* a);
hipError_t launch_diff_bwd(const DiffBwd& a, hipStream_t stream);

}  // namespace sol
