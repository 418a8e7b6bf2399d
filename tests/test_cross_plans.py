"""How cross attention and the norm and rotation's gradients cut their calls (CPU
only): the plans of libsol.so, called from a small program over many shapes.  Pieces
have keys and fit the heads and rows that they divide, the workspace's sections lie
one after the other inside it, and no launch passes 2^32 threads."""
import os
import shutil
import subprocess

import pytest

from paper_2609_35110_amd import build as pkg_build
from paper_2609_35110_amd import sol

SRC = r"""
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include "sol.h"
#include "sol_cross.h"
using namespace sol;

#define CHECK(x)                                                                                                   \
  do {                                                                                                             \
    if (!(x)) {                                                                                                    \
      printf("%s: B=%d H=%d Hk=%d N=%d M=%d masked=%d (line %d)\n", #x, s.B, s.H, s.Hk, s.N, s.M, s.mask != nullptr, \
             __LINE__);                                                                                            \
      exit(1);                                                                                                     \
    }                                                                                                              \
  } while (0)

static int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
static const int64_t kThreads = (int64_t)1 << 32;

static void norm_rope(const CrossShape& s) {
  const int64_t need = norm_rope_bwd_bytes((int64_t)s.B * s.N, s.H + s.Hk);
  CHECK(need >= 1024 && need % 1024 == 0 && need / 1024 <= std::max(2 * 2048, s.H + s.Hk));
  const bool taken = (int64_t)s.B * s.N <= ((int64_t)1 << 28) - 16 && s.H + s.Hk < 1 << 16;
  CHECK((int64_t)sol_qk_norm_rope_bwd_workspace_bytes(s.B, s.H, s.Hk, s.N, 128) == (taken ? need : 0));
}

static bool few, brief, split, pieces, masked_tiles, large;
static void fwd(const CrossShape& s) {
  const int64_t tiles = (int64_t)s.B * s.H * up(s.N, kCrossRows), turns = up(s.M, 32);
  const int64_t got = cross_fwd_bytes(s, nullptr, nullptr);
  const int64_t order = s.mask && s.M > kShortKeys ? up(((int64_t)s.B * s.M + s.B) * 4, 256) * 256 : 0;
  for (bool ragged : {false, true}) {
    const CrossPlan p = cross_plan(s, ragged);
    if (p.few) {
      const int64_t groups = up((int64_t)(s.H / s.Hk) * s.N, kFewRows);
      CHECK(p.pieces >= 1 && (p.pieces == 1 || s.M / p.pieces >= 512));
      if (got == (int64_t)kTooLarge) continue;
      CHECK((int64_t)s.B * s.Hk * p.pieces * groups * 512 < kThreads);
      if (p.pieces > 1) {
        CHECK(got >= (int64_t)s.B * s.H * s.N * p.pieces * (128 + 2) * 4);  // o, the sums and the exact ones
        CHECK((int64_t)s.B * s.H * s.N * 256 < kThreads);
      }
      few = true;
      pieces |= p.pieces > 1;
    } else {
      CHECK(p.brief == (s.M <= kShortKeys) && !(p.brief && p.split));
      // every workgroup has a turn: a share that is joined is one that was written
      CHECK(p.workgroups >= 1 && p.workgroups <= kCus && p.workgroups <= (p.brief ? tiles : tiles * turns));
      if (p.brief) {
        CHECK(got == 0);
        brief = true;
        continue;
      }
      if (got == (int64_t)kTooLarge) { large = true; continue; }
      CHECK(got >= order + (p.split ? (int64_t)2 * p.workgroups * kCrossRows * (128 + 2) * 4 : 0));
      CHECK(tiles * (kCrossRows / 16) * 256 < kThreads && (int64_t)s.B * 1024 < kThreads);
      split |= p.split;
      masked_tiles |= s.mask != nullptr;
    }
  }
  const int64_t told = sol_cross_attn_fwd_workspace_bytes(s.B, s.H, s.Hk, s.N, s.M, 128, s.mask != nullptr);
  CHECK(told == (got == (int64_t)kTooLarge ? 0 : got));
  if (got == (int64_t)kTooLarge || cross_plan(s, true).few || cross_plan(s, true).brief) return;
  CrossFwd a = {};
  char* at = reinterpret_cast<char*>(1 << 20);
  CHECK((int64_t)cross_fwd_bytes(s, &a, at) == got);
  CHECK(reinterpret_cast<char*>(a.ws) == at + order);
  if (s.mask) CHECK(reinterpret_cast<char*>(a.order) == at && a.counts == a.order + (int64_t)s.B * s.M);
}

static bool head_pieces, row_pieces, cut, brief_parts;
static void bwd(const CrossShape& s) {
  CrossBwd a = {};
  char* at = reinterpret_cast<char*>(1 << 20);
  const int64_t got = cross_bwd_bytes(s, &a, at);
  const int64_t told = sol_cross_attn_bwd_workspace_bytes(s.B, s.H, s.Hk, s.N, s.M, 128, s.mask != nullptr);
  CHECK(told == (got == (int64_t)kTooLarge ? 0 : got));
  const bool always = (int64_t)s.B * s.H * s.N <= 1 << 25 && (int64_t)s.B * s.Hk * s.M <= 1 << 25 && (int64_t)s.B * s.H <= 1 << 20;
  if (always) CHECK(got != (int64_t)kTooLarge && (int64_t)cross_fwd_bytes(s, nullptr, nullptr) != (int64_t)kTooLarge);
  if (got == (int64_t)kTooLarge) return;
  CHECK((int64_t)cross_bwd_bytes(s, nullptr, nullptr) == got);
  const int64_t slabs = (int64_t)s.B * s.Hk, blocks = (s.H / s.Hk) * up(s.N, 32);
  if (s.M <= kCrossKeys && (slabs >= 8 || blocks <= 64)) {  // a key head's rows in parts, which have blocks of 32
    const int64_t parts = a.row_pieces;
    CHECK(a.head_pieces == 1 && parts >= 1 && parts <= blocks && (parts == 1 || slabs * parts <= kCus));
    CHECK(a.plan.full == (int64_t)s.B * s.H * up(s.N, kCrossRows) && a.plan.pieces == 1);
    CHECK(got == (parts > 1 ? slabs * parts * 2 * kCrossKeys * 128 * 4 : 0) && slabs * parts * 256 < kThreads);
    CHECK(reinterpret_cast<char*>(a.dkv_parts) == at);
    brief_parts |= parts > 1;
    return;
  }
  const int64_t tiles = (int64_t)s.B * s.H * up(s.N, kCrossRows), rest = tiles - a.plan.full;
  CHECK(rest >= 0 && a.plan.full >= 0 && a.plan.pieces >= 1);
  if (a.plan.pieces == 1) CHECK(rest == 0);
  else CHECK(a.plan.pieces <= 32 && s.M / a.plan.pieces >= 64);
  const int64_t key_tiles = (int64_t)s.B * s.Hk * up(s.M, kCrossKeys), all = (int64_t)a.head_pieces * a.row_pieces;
  CHECK(a.head_pieces >= 1 && a.row_pieces >= 1 && (s.H / s.Hk) % a.head_pieces == 0);
  if (a.row_pieces > 1) CHECK(a.head_pieces == s.H / s.Hk && s.N / a.row_pieces >= 256);
  const int64_t groups = (int64_t)s.B * s.H * up(s.N, 32);
  const char* end = at + got;
  struct { const void* p; int64_t bytes; } sections[] = {
      {at, s.mask ? ((int64_t)s.B * s.M + s.B) * 4 : 0},
      {a.stats, groups * 64 * 4},
      {a.dq_parts, a.plan.pieces > 1 ? rest * a.plan.pieces * kCrossRows * 128 * 4 : 0},
      {a.dkv_parts, all > 1 ? key_tiles * all * 2 * kCrossKeys * 128 * 4 : 0}};
  for (auto& x : sections) {
    const char* p = static_cast<const char*>(x.p);
    CHECK(p >= at && reinterpret_cast<uintptr_t>(p) % 256 == 0);
    at = const_cast<char*>(p) + x.bytes;
  }
  CHECK(at <= end);
  if (s.mask) CHECK(a.counts == a.order + (int64_t)s.B * s.M);
  CHECK(groups * 512 < kThreads);
  CHECK((key_tiles * all + a.plan.full + rest * a.plan.pieces) * 256 < kThreads);
  CHECK((rest * 16 + (all > 1 ? key_tiles * 16 : 0)) * 256 < kThreads);
  head_pieces |= a.head_pieces > 1;
  row_pieces |= a.row_pieces > 1;
  cut |= a.plan.pieces > 1;
}

int main() {
  static const uint8_t some = 1;
  std::mt19937_64 rng(1);
  auto log = [&](double lo, double hi) {
    return (int)std::lround(std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi))(rng)));
  };
  for (int n = 0; n < 200000; ++n) {
    CrossShape s = {};
    const bool wide = n % 8 == 0;
    s.B = log(1, wide ? 1 << 16 : 64);
    s.Hk = log(1, wide ? 1 << 12 : 48);
    s.H = s.Hk * log(1, wide ? 300 : 16);
    s.N = log(1, n % 3 ? 150000 : 8 << 20);
    s.M = log(1, n % 5 ? 4096 : 8 << 20);
    if (n % 4 == 1) s.N = log(1, 200);
    s.scale = 1.0f;
    s.mask = rng() & 1 ? &some : nullptr;
    norm_rope(s);
    if ((int64_t)s.B * s.H > 1 << 22 || (int64_t)s.B * s.H * s.N > INT32_MAX || (int64_t)s.B * s.Hk * s.M > INT32_MAX) continue;
    fwd(s);
    bwd(s);
  }
  printf("few %d brief %d pieces %d split %d masked tiles %d head pieces %d row pieces %d cut %d large %d\n", few, brief, pieces, split, masked_tiles,
         head_pieces, row_pieces, cut, large);
  if (!(few && brief && pieces && split && masked_tiles && head_pieces && row_pieces && cut && brief_parts && large)) return 1;  // each kind was met
  puts("plans hold");
}
"""


def test_plans_hold(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("g++ or the HIP headers not available")
    if not os.path.exists(sol.LIB_PATH):
        pkg_build.build()
    src, exe = str(tmp_path / "plans.cpp"), str(tmp_path / "plans")
    open(src, "w").write(SRC)
    pkg = os.path.dirname(sol.LIB_PATH)
    res = subprocess.run([gxx, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", pkg_build.INCLUDE,
                          "-I", pkg_build.CSRC, src, "-o", exe, "-L", pkg, "-l:libsol.so", "-L/opt/rocm/lib", "-lamdhip64",
                          "-Wl,-rpath," + pkg + ":/opt/rocm/lib"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "plans hold" in res.stdout, res.stdout + res.stderr
