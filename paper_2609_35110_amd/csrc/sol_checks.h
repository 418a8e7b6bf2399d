// Checks of arguments that the C ABI's front ends share (sol_api_ops.cpp,
// sol_api_cross.cpp): strided rows, spans that may not meet, workspaces.  Host
// only, before any HIP call.
#pragma once

#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "sol.h"
#include "sol_ops.h"

namespace {

inline int fail(int status, const char* fmt, ...) {
  char msg[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof msg, fmt, ap);
  va_end(ap);
  return sol::set_error(status, msg);
}

inline int done(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(SOL_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
  return sol::set_error(SOL_OK, "");
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A piece of memory that a call reads or writes: all of its bytes, or rows of D
// elements in it (strides s and counts n, in elements).
struct Span {
  const char* name;
  uintptr_t at;
  uint64_t bytes;
  bool rows;
  int64_t s[3], n[3];
};
inline Span span(const char* name, const void* p, uint64_t bytes) {
  return {name, reinterpret_cast<uintptr_t>(p), p ? bytes : 0, false, {}, {}};
}
// What rows cover of every `period` elements from their first on, 0 where that is
// no bound: the strides that are no multiple of it are to stay within one.
inline int64_t covered(const Span& x, int64_t period) {
  int64_t last = 0;
  for (int i = 0; i < 3; ++i) {
    if (x.n[i] == 1 || x.s[i] % period == 0) continue;
    if (x.s[i] > period || x.n[i] - 1 > period / x.s[i]) return 0;
    last += (x.n[i] - 1) * x.s[i];
  }
  return last + sol::kHeadDim <= period ? last + sol::kHeadDim : 0;
}
// Rows side by side in one buffer, as of a packed q, k and v: seen modulo a stride
// of either, neither's part of a period meets the other's.
inline bool side_by_side(const Span& x, const Span& y) {
  if (!x.rows || !y.rows) return false;
  for (int i = 0; i < 6; ++i) {
    const int64_t period = i < 3 ? x.s[i] : y.s[i - 3];
    if ((i < 3 ? x.n[i] : y.n[i - 3]) == 1 || period == 0) continue;
    const int64_t cx = covered(x, period), cy = covered(y, period);
    if (!cx || !cy) continue;
    int64_t from = (static_cast<int64_t>(y.at - x.at) / 2) % period;  // (both are 16-byte aligned)
    if (from < 0) from += period;
    if (from >= cx && from + cy <= period) return true;
  }
  return false;
}
inline bool meet(const Span& x, const Span& y) {
  return x.bytes && y.bytes && x.at < y.at + y.bytes && y.at < x.at + x.bytes && !side_by_side(x, y);
}

constexpr int64_t kMaxStride = (int64_t)1 << 40;
// Elements between tokens: the kernels' copies address the rows of a tile by 32-bit byte offsets.
constexpr int64_t kMaxRowStride = (int64_t)1 << 24;

// The rows of one tensor: its strides (contiguous when null) checked, its span
// found.  An output's rows must not meet: from the finest dimension up, each
// stride has to pass what the finer ones cover.
inline int take_rows(const char* name, const void* p, const sol_strides* st, int B, int H, int N, bool out, sol::Rows* rows,
              Span* sp) {
  const int64_t D = sol::kHeadDim;
  if (!p) return fail(SOL_ERR_INVALID_ARG, "%s must not be NULL", name);
  if (!aligned16(p)) return fail(SOL_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
  const int64_t s[3] = {st ? st->b : (int64_t)H * N * D, st ? st->h : (int64_t)N * D, st ? st->n : D};
  const int64_t n[3] = {B, H, N};
  uint64_t last = 0;
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) continue;  // a stride that is never taken
    if (s[i] < 0 || s[i] % 8 || s[i] > kMaxStride)
      return fail(SOL_ERR_INVALID_ARG, "%s strides must be non-negative multiples of 8 elements (got %lld, %lld, %lld)",
                  name, (long long)s[0], (long long)s[1], (long long)s[2]);
    if (i == 2 && s[i] > kMaxRowStride)
      return fail(SOL_ERR_UNSUPPORTED, "%s: %lld elements between tokens (at most 2^24)", name, (long long)s[i]);
    last += (uint64_t)(n[i] - 1) * (uint64_t)s[i];
  }
  if (out) {
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 2; ++i)
      for (int j = 0; j < 2 - i; ++j)
        if (s[order[j]] > s[order[j + 1]]) {
          const int t = order[j];
          order[j] = order[j + 1];
          order[j + 1] = t;
        }
    uint64_t covered = D;
    for (int i : order) {
      if (n[i] == 1) continue;
      if ((uint64_t)s[i] < covered) return fail(SOL_ERR_INVALID_ARG, "rows of %s overlap each other", name);
      covered += (uint64_t)(n[i] - 1) * (uint64_t)s[i];
    }
  }
  rows->p = static_cast<uint16_t*>(const_cast<void*>(p));
  rows->sb = B == 1 ? 0 : s[0];
  rows->sh = H == 1 ? 0 : s[1];
  rows->sn = N == 1 ? 0 : s[2];
  *sp = {name, reinterpret_cast<uintptr_t>(p), (last + D) * 2, true, {s[0], s[1], s[2]}, {n[0], n[1], n[2]}};
  return SOL_OK;
}

// No output may meet an input or another output.
inline int check_apart(const Span* in, int n_in, const Span* out, int n_out) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (meet(out[i], in[j])) return fail(SOL_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, in[j].name);
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return fail(SOL_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, out[j].name);
  }
  return SOL_OK;
}

inline int check_heads(int B, int H, int Hk, int N, int D) {
  if (B < 1 || H < 1 || Hk < 1 || N < 1)
    return fail(SOL_ERR_INVALID_ARG, "B, H, Hk, N must be >= 1 (got %d, %d, %d, %d)", B, H, Hk, N);
  if (H % Hk) return fail(SOL_ERR_INVALID_ARG, "H = %d is not a multiple of Hk = %d", H, Hk);
  if (D != sol::kHeadDim) return fail(SOL_ERR_UNSUPPORTED, "head dim %d not supported (only 128)", D);
  if (N > SOL_MAX_TOKENS) return fail(SOL_ERR_UNSUPPORTED, "N=%d exceeds %d", N, SOL_MAX_TOKENS);
  return SOL_OK;
}

// A small array of the device: 4-byte aligned.
inline int check_small(const char* name, const void* p, bool may_be_null) {
  if (!p) return may_be_null ? SOL_OK : fail(SOL_ERR_INVALID_ARG, "%s must not be NULL", name);
  if (reinterpret_cast<uintptr_t>(p) & 3u) return fail(SOL_ERR_INVALID_ARG, "%s must be 4-byte aligned", name);
  return SOL_OK;
}

inline int check_workspace(const void* ws, size_t bytes, size_t need) {
  if (!need) return SOL_OK;
  if (!ws) return fail(SOL_ERR_INVALID_ARG, "workspace is NULL");
  if (!aligned16(ws)) return fail(SOL_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  if (bytes < need) return fail(SOL_ERR_INVALID_ARG, "workspace needs %zu bytes, got %zu", need, bytes);
  return SOL_OK;
}

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

#define SOL_TRY(x)                    \
  do {                                \
    const int st_ = (x);              \
    if (st_ != SOL_OK) return st_;    \
  } while (0)

}  // namespace
