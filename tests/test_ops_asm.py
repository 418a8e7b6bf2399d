"""Checks on the generated gfx950 code of the linear and differential attention's
kernels (CPU only), whose score MFMAs and tile copies are inline assembly that the
compiler's hazard recognizer does not see: MFMA latencies, operands settled
before an inline MFMA, no spills (a reload's wait would wait for the copies
too), M0 used by the copies alone, and no wait for the copies but the ones
written beside the barriers."""
import os
import re
import shutil
import subprocess

import pytest

import test_kernel_asm as checks
from paper_2609_35110_amd import build as pkg_build

# (source, {kernel: instances}): maps on one key head or on one each, the forward
# kernel also for training or not
SOURCES = [("sol_diff_attn.hip", {"diff_fwd_kernel": 4, "diff_bwd_kernel": 2}),
           ("sol_lin_attn.hip", {"lin_state_kernel": 1, "lin_scan_kernel": 1})]
WRITE_WAIT_STATES = 2  # a VALU write of an MFMA's A, B or C operand


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    flags = [f for f in pkg_build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    found = []
    for source, names in SOURCES:
        out = str(tmp_path_factory.mktemp("asm") / (source + ".s"))
        src = os.path.join(pkg_build.CSRC, source)
        res = subprocess.run([hipcc] + flags + ["--cuda-device-only", "-S", "-I", pkg_build.INCLUDE, "-I",
                                                pkg_build.CSRC, "-x", "hip", src, "-o", out],
                             capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-2000:]
        text = open(out).read()
        for name in names:
            instances = checks.functions(text, name)
            assert len(instances) == names[name], name
            found += instances
    # (the state's kernel alone has fewer MFMAs than a listing is expected to have)
    lin = [f for f in found if "lin_" in f[0]]
    return [f for f in found if f not in lin] + [("lin kernels", sum((body for _, body in lin), []))]


def test_mfma_latency(kernels):
    """No instruction reads or overwrites an MFMA's result, or overwrites its
    accumulator input, within the 12 wait states it needs, chained MFMAs aside
    (inline MFMAs and the compiler's own)."""
    checks.check_mfma_latency(kernels, past_branches=False)


def test_no_spills(kernels):
    checks.check_no_spills(kernels)


def test_operands_settled_before_inline_mfmas(kernels):
    for name, body in kernels:
        ins = checks.instructions(body)
        for i, (t, in_asm) in enumerate(ins):
            if not (in_asm and t.startswith("v_mfma")):
                continue
            used = set().union(*(checks.regs(o) for o in checks.operands(t)[1:]))
            ws = 0
            for t2, _ in reversed(ins[max(0, i - 20):i]):
                if ws >= WRITE_WAIT_STATES:
                    break
                if t2.startswith("v_") and not t2.startswith("v_mfma") and checks.operands(t2):
                    assert not (checks.regs(checks.operands(t2)[0]) & used), "%s: %r then %r" % (name, t2, t)
                m = re.match(r"s_nop (\d+)", t2)
                ws += int(m.group(1)) + 1 if m else 1


def test_m0_used_only_by_copies(kernels):
    for name, body in kernels:
        ins = checks.instructions(body)
        sets = [i for i, (t, _) in enumerate(ins) if re.search(r"\bm0\b", t)]
        assert sets
        for i in sets:
            assert ins[i][1] and ins[i][0].startswith("s_mov_b32 m0"), "%s: %r" % (name, ins[i][0])
            assert ins[i + 1][0] == "s_nop 0" and ins[i + 2][0].startswith("global_load_lds_"), name


def test_copies_are_waited_for_only_at_the_barriers(kernels):
    """In the loops (between an inline wait and the next) no other wait drains
    the copies on their way: a vmcnt wait of the compiler's stands only where a
    load of its own is used, outside the turns."""
    for name, body in kernels:
        if "diff" not in name:
            continue
        blocks, cur = [], []
        for ln in body:
            if re.match(r"\.LBB", ln):
                blocks.append(cur)
                cur = []
            cur.append(ln)
        blocks.append(cur)
        turns = [b for b in blocks if sum("v_exp_f32" in ln for ln in b) >= 8 and sum("v_mfma" in ln for ln in b) >= 8]
        assert len(turns) >= (4 if "bwd" in name else 2), name
        for b in turns:
            for t, in_asm in checks.instructions(b):
                assert in_asm or "vmcnt" not in t, "%s: %r" % (name, t)


def test_copy_sgprs_not_written_by_valu_just_before(kernels):
    """A vector-memory instruction reading an SGPR that a VALU instruction wrote
    needs 5 wait states between them (see the prepared-path kernel's check)."""
    for name, body in kernels:
        ins = checks.instructions(body)
        for i, (t, in_asm) in enumerate(ins):
            if not t.startswith("global_load_lds_"):
                continue
            used = set().union(*(checks.sregs(o) for o in checks.operands(t)))
            assert used, "%s: %r" % (name, t)
            ws = 0
            for t2, _ in reversed(ins[max(0, i - 40):i]):
                m = re.match(r"s_nop (\d+)", t2)
                ws += int(m.group(1)) + 1 if m else 1
                if ws > 5:
                    break
                if t2.startswith("v_") and checks.operands(t2):
                    assert not (checks.sregs(checks.operands(t2)[0]) & used), "%s: %r then %r" % (name, t2, t)
