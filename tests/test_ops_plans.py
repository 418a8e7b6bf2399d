"""How the linear and differential attention cut their calls (CPU only): the plans
of libsol.so, called from a small program over many shapes.  Segments, tiles and
pieces cover each token, row and key once and none is empty, the workspace's
sections lie one after the other inside it, and no launch passes 2^32 threads."""
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
#include "sol_ops.h"
using namespace sol;

#define CHECK(x)                                                                                                  \
  do {                                                                                                            \
    if (!(x)) {                                                                                                   \
      printf("%s: B=%d H=%d Hv=%d Hk=%d N=%d M=%d causal=%d (line %d)\n", #x, s.B, s.H, s.Hv, s.Hk, s.N, s.M,     \
             s.causal, __LINE__);                                                                                 \
      exit(1);                                                                                                    \
    }                                                                                                             \
  } while (0)

static int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

static void lin(const DiffShape& s) {  // (B, H, N)
  const int64_t slabs = (int64_t)s.B * s.H;
  for (int scans : {1, 3}) {
    const LinPlan p = lin_plan(slabs, s.N, scans);
    CHECK(p.parts >= 1 && p.nseg >= 1 && p.seg_rows > 0);
    CHECK(p.seg_rows % (kLinRows * p.parts) == 0);                   // parts of whole chunks
    CHECK((int64_t)p.nseg * p.seg_rows >= s.N);                      // every token is in a segment
    CHECK((int64_t)(p.nseg - 1) * p.seg_rows < s.N);                 // and every segment has one
    CHECK((int64_t)p.nseg * p.seg_rows < INT32_MAX);
    const int64_t sets = scans > 1 ? 2 : 1;
    const int64_t need = p.nseg > 1 ? slabs * p.nseg * p.parts * sets * kStateElems * 4 : 0;
    CHECK((int64_t)lin_states_bytes(slabs, s.N, scans) == need);
    CHECK(slabs * p.nseg * scans * 512 < (int64_t)1 << 32);
    if (p.nseg > 1) {
      CHECK(slabs * p.nseg * p.parts * sets * 512 < (int64_t)1 << 32);
      CHECK(slabs * p.nseg <= 512);  // (segments are for calls of few slabs)
    }
  }
  CHECK((int64_t)sol_lin_attn_fwd_workspace_bytes(s.B, s.H, s.N, 128) == (int64_t)lin_states_bytes(slabs, s.N, 1));
  const int64_t part = s.Hv < s.H ? 2 * slabs * s.N * 128 * 4 : 0;
  const int64_t all = sol_lin_attn_bwd_workspace_bytes(s.B, s.H, s.Hv, s.N, 128);
  if (part && (int64_t)s.B * s.Hv * s.N > 1 << 26) CHECK(all == 0);
  else CHECK(all >= (int64_t)lin_states_bytes(slabs, s.N, 3) + part);
}

static void tiles_whole_or_cut(const DiffShape& s, int64_t tiles, const DiffTiles& t) {
  CHECK(t.full >= 0 && t.full <= tiles && t.pieces >= 1);
  if (t.pieces == 1) CHECK(t.full == tiles);
  else CHECK(t.pieces <= 16 && s.M / t.pieces >= 512);
}

static void diff(const DiffShape& s) {
  const int64_t rows = (int64_t)s.B * s.H * s.N, tiles = (int64_t)s.B * s.H * up(s.N, kDiffRows);
  const int64_t got = diff_fwd_bytes(s);
  for (bool ragged : {false, true}) {
    const DiffPlan p = diff_plan(s, ragged);
    int64_t joined, workgroups;
    if (p.few) {
      const int64_t groups = up((int64_t)(s.H / s.Hv) * s.N, kFewRows);
      CHECK(s.N <= kDiffRows && p.tiles.full == 0 && p.tiles.pieces >= 1);
      CHECK(p.tiles.pieces == 1 || s.M / p.tiles.pieces >= 128);
      joined = p.tiles.pieces > 1 ? rows : 0;
      workgroups = up((int64_t)s.B * s.Hv * p.tiles.pieces, 8) * 8 * groups;
    } else {
      tiles_whole_or_cut(s, tiles, p.tiles);
      joined = (tiles - p.tiles.full) * kDiffRows;
      workgroups = p.tiles.full + (tiles - p.tiles.full) * p.tiles.pieces;
    }
    if (got == (int64_t)kTooLarge) continue;
    CHECK(workgroups * 256 < (int64_t)1 << 32);
    CHECK(got >= joined * p.tiles.pieces * 2 * (128 + 2) * 4);  // o, the sums and the exact ones, of both maps
    CHECK((p.few ? joined : joined / 4) * 256 < (int64_t)1 << 32);
  }
  if (got != (int64_t)kTooLarge) CHECK((int64_t)sol_diff_attn_fwd_workspace_bytes(s.B, s.H, s.Hv, s.N, s.M, 128) >= got);

  DiffBwd a = {};
  a.s = s;
  a.stats = reinterpret_cast<float*>(1 << 20);
  const int64_t bytes = diff_bwd_bytes(s, &a);
  if (bytes == (int64_t)kTooLarge) return;
  CHECK((int64_t)sol_diff_attn_bwd_workspace_bytes(s.B, s.H, s.Hv, s.N, s.M, 128) >= bytes);
  tiles_whole_or_cut(s, tiles, a.plan);
  const int64_t key_tiles = (int64_t)s.B * s.Hv * up(s.M, kDiffRows), pieces = (int64_t)a.head_pieces * a.row_pieces;
  CHECK(a.head_pieces >= 1 && a.row_pieces >= 1 && (s.H / s.Hv) % a.head_pieces == 0);
  if (a.row_pieces > 1) CHECK(a.head_pieces == s.H / s.Hv && s.N / a.row_pieces >= 256);
  CHECK(a.parts == 4 * up(s.M, kDiffRows) * a.row_pieces);
  const char* at = reinterpret_cast<char*>(a.stats);
  const int64_t groups = (int64_t)s.B * s.H * up(s.N, 32);
  struct { const float* p; int64_t floats; } sections[] = {
      {a.stats, groups * 128}, {a.delta, groups}, {a.partial, (int64_t)s.H * s.B * a.parts},
      {a.dq_parts, a.plan.pieces > 1 ? (tiles - a.plan.full) * a.plan.pieces * 2 * kDiffRows * 128 : 0},
      {a.dkv_parts, pieces > 1 ? key_tiles * pieces * 3 * kDiffRows * 128 : 0}};
  for (auto& x : sections) {
    const char* p = reinterpret_cast<const char*>(x.p);
    CHECK(p >= at && reinterpret_cast<uintptr_t>(p) % 16 == 0);
    at = p + x.floats * 4;
  }
  CHECK(at <= reinterpret_cast<char*>(a.stats) + bytes);
  CHECK(groups * 512 < (int64_t)1 << 32);
  CHECK((key_tiles * pieces + a.plan.full + (tiles - a.plan.full) * a.plan.pieces) * 256 < (int64_t)1 << 32);
  CHECK((s.H + (tiles - a.plan.full) * 16 + (pieces > 1 ? key_tiles * 24 : 0)) * 256 < (int64_t)1 << 32);
}

int main() {
  std::mt19937_64 rng(1);
  auto log = [&](double lo, double hi) {
    return (int)std::lround(std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi))(rng)));
  };
  int n = 0, cut = 0, few = 0, keys = 0, segments = 0;
  while (n < 200000) {
    DiffShape s = {};
    const bool wide = n % 8 == 0;
    s.B = log(1, wide ? 1 << 16 : 64);
    s.Hv = log(1, wide ? 1 << 12 : 48);
    s.H = s.Hv * log(1, wide ? 300 : 16);
    s.N = log(1, n % 3 ? 150000 : 8 << 20);
    s.M = log(1, n % 5 ? 150000 : 8 << 20);
    if (n % 4 == 1) s.N = log(1, 200);
    if (n % 7 == 2) s.M = s.N;
    s.Hk = s.Hv * (1 + (int)(rng() & 1));
    s.causal = (int)(rng() & 1);
    s.scale = 1.0f;
    ++n;
    if ((int64_t)s.B * s.H <= 1 << 21) {
      lin(s);
      segments += lin_plan((int64_t)s.B * s.H, s.N, 1).nseg > 1;
    }
    if ((int64_t)s.B * s.H > 1 << 22 || (int64_t)s.B * s.H * s.N > INT32_MAX || (int64_t)s.B * s.Hv * s.M > INT32_MAX) continue;
    diff(s);
    const DiffPlan p = diff_plan(s, false);
    DiffBwd a = {};
    a.s = s;
    diff_bwd_bytes(s, &a);
    few += p.few;
    cut += p.tiles.pieces > 1;
    keys += a.head_pieces * a.row_pieces > 1;
  }
  printf("few %d cut %d key pieces %d segments %d\n", few, cut, keys, segments);
  // each kind was met
  if (few < 1000 || cut < 1000 || keys < 1000 || segments < 1000) return 1;
  puts("plans hold");
}
"""


def test_plans_cover_every_row_and_key(tmp_path):
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
