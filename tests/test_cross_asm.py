"""Checks on the generated gfx950 code of cross attention's kernels (CPU only), whose
score MFMAs and tile copies are inline assembly that the compiler's hazard recognizer
does not see: MFMA latencies, operands settled before an inline MFMA, no spills, M0
used by the copies alone -- and, since the forward kernel's turns wait for copies by
the number of the wave's memory operations after them, that number as it is written."""
import os
import re
import shutil
import subprocess

import pytest

import test_kernel_asm as checks
import test_ops_asm as ops
from paper_2609_35110_amd import build as pkg_build

NAMES = {"cross_fwd_kernel": 4, "cross_bwd_kernel": 2}  # instances: masked or not, the forward ones for training or not


@pytest.fixture(scope="module")
def text(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    out = str(tmp_path_factory.mktemp("asm") / "cross.s")
    flags = [f for f in pkg_build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    src = os.path.join(pkg_build.CSRC, "sol_cross_attn.hip")
    res = subprocess.run([hipcc] + flags + ["--cuda-device-only", "-S", "-I", pkg_build.INCLUDE, "-I", pkg_build.CSRC,
                                            "-x", "hip", src, "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    return open(out).read()


@pytest.fixture(scope="module")
def kernels(text):
    found = []
    for name, n in NAMES.items():
        instances = checks.functions(text, name)
        assert len(instances) == n, name
        found += instances
    # (few keys' backward kernel alone has fewer inline MFMAs than a listing is expected to have)
    short = checks.functions(text, "cross_short_bwd_kernel")
    assert len(short) == 1
    return found + [("few keys' gradients, and cross_bwd_kernel", short[0][1] + found[-1][1])]


def test_mfma_latency(kernels):
    checks.check_mfma_latency(kernels, past_branches=False)


def test_no_spills(kernels, text):
    checks.check_no_spills(kernels)
    for name, n in (("cross_short_kernel", 8), ("cross_short_bwd_kernel", 1), ("cross_few_kernel", 2)):
        instances = checks.functions(text, name)
        assert len(instances) == n, name
        checks.check_no_spills(instances)


def test_operands_settled_before_inline_mfmas(kernels):
    ops.test_operands_settled_before_inline_mfmas(kernels)


def test_m0_used_only_by_copies(kernels):
    ops.test_m0_used_only_by_copies(kernels)


def test_copy_sgprs_not_written_by_valu_just_before(kernels):
    for name, body in kernels:  # (masked keys' copies have their addresses in VGPRs alone)
        with_sgprs = [ln for ln in body if not re.match(r"\s*global_load_lds_\w+ v\[\d+:\d+\], off\b", ln)]
        ops.test_copy_sgprs_not_written_by_valu_just_before([(name, with_sgprs)])


def blocks(body):
    """The instructions of each basic block."""
    found, cur = [], []
    for ln in body:
        if re.match(r"(\.LBB|; %bb)", ln):
            found.append(cur)
            cur = []
        cur.append(ln)
    return [checks.instructions(b) for b in found + [cur]]


def count(block, start):
    return sum(t.startswith(start) for t, _ in block)


def forward(kernels):
    """(name, masked, training, blocks) of the forward kernel's instances."""
    for name, body in kernels:
        m = re.search(r"cross_fwd_kernelILb(\d)ELb(\d)E", name)
        if m:
            yield name, m.group(1) == "1", m.group(2) == "1", blocks(body)


def test_turns_wait_by_count_alone(kernels):
    """A turn's only waits for memory are the counted ones (two turns' copies, and in a
    tile's first three the rows' operations): the compiler has none of its own beside its
    MFMAs, whose loads would have it wait for the copies on their way."""
    for name, _, training, found in forward(kernels):
        turns = [b for b in found if count(b, "v_exp_f32") >= 30 and count(b, "v_mfma") >= 28]
        assert len(turns) == 2, name
        for b in turns:
            assert count(b, "global_load_lds_dwordx4") == 4 and not count(b, "global_load_dword"), name
            assert not [t for t, in_asm in b if "vmcnt" in t and not in_asm], name
        # the waits: 8, or the rows' too
        inline = [int(m.group(1)) for b in found for t, in_asm in b if in_asm for m in [re.match(r"s_waitcnt vmcnt\((\d+)\)$", t)] if m]
        assert sorted(set(inline)) == [0, 8, 12, 8 + (50 if training else 32)], name


def test_rows_operations_as_counted(kernels):
    """A tile's end is 16 stores of a wave's output (for training twice 16 and two of the
    log sums) in straight lines, and the next rows' copies are 16."""
    for name, _, training, found in forward(kernels):
        copies = [b for b in found if count(b, "global_load_lds_dwordx4") == 16]
        assert len(copies) == 2, name  # the first tile's, and a later one's
        staged = [b for b in found if count(b, "ds_write") and count(b, "global_store_dwordx4") >= 16]
        assert len(staged) == 1, name
        assert count(staged[0], "global_store_dwordx4") == (32 if training else 16), name
        assert not count(staged[0], "global_load"), name


def test_backward_turns_wait_at_their_marks(kernels):
    """Between a wait that the source has and the next no other one drains the copies."""
    for name, body in kernels:
        if "cross_bwd_kernelILb" not in name:
            continue
        turns = [b for b in blocks(body) if count(b, "v_exp_f32") >= 5 and count(b, "v_mfma") >= 8]
        assert len(turns) >= 4, name
        for b in turns:
            assert not [t for t, in_asm in b if "vmcnt" in t and not in_asm], name
