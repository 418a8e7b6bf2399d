"""The largest calls of cross attention, by what the front end says (CPU only): what
include/sol.h says is always taken is, at its bounds too, and a limit of a launch that
a call does not make refuses nothing."""
import pytest

from paper_2609_35110_amd import sol
from test_cross_abi import at, cross_bwd, cross_fwd

TOO_LARGE = "too large together"


def said(status, fragment):
    """Which of a call's refusals comes: each call here has an output over an input besides, found after its size."""
    assert status != 0
    return fragment in sol.sol_last_error()


def taken(B, H, Hk, N, M, masked):
    """(forwards, backwards): not refused for its size."""
    sizes = dict(B=B, H=H, Hk=Hk, N=N, M=M, mask=at(7) if masked else None, q=1 << 44, k=1 << 45, v=1 << 46, out=1 << 47,
                 left=1 << 48, lse=1 << 49, ws=1 << 50, ws_bytes=1 << 50)
    fwd = cross_fwd(**dict(sizes, left=sizes["q"]))
    fwd = not said(fwd, TOO_LARGE) and said(fwd, "out_left overlaps q")
    bwd = cross_bwd(**dict(sizes, dout=1 << 51, dq=sizes["q"], dk=1 << 52, dv=1 << 53))
    bwd = not said(bwd, TOO_LARGE) and said(bwd, "dq overlaps q")
    ask = (B, H, Hk, N, M, 128, int(masked))
    if not fwd:
        assert sol.sol_cross_attn_fwd_workspace_bytes(*ask) == 0
    if not bwd:
        assert sol.sol_cross_attn_bwd_workspace_bytes(*ask) == 0
    return fwd, bwd


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("heads", [1, 4, 64, 1 << 10, 1 << 16, 1 << 20])  # of the 2^20 slabs, a sequence's
def test_what_is_always_taken(heads, masked):
    B = (1 << 20) // heads
    for Hk in {1, heads // 2 or 1, heads}:
        for N in (1, 2, 31, 32):
            for M in {1, 128, 129, 256, 257, 512, min((1 << 25) // (B * Hk), 1 << 23)}:
                if B * Hk * M <= 1 << 25:
                    assert taken(B, heads, Hk, N, M, masked) == (True, True), (B, heads, Hk, N, M)


def test_row_tiles():
    assert taken(1 << 14, 64, 1, 256, 512, False)[0] and taken(1 << 10, 64, 64, 16 * 256, 300, True)[0]
    assert not taken(1 << 14, 64, 1, 257, 512, False)[0] and not taken((1 << 14) + 1, 64, 1, 256, 512, False)[0]
    # few rows, or few keys, run otherwise
    assert taken(1 << 16, 64, 2, 1, 512, False)[0] and taken(1 << 14, 64, 1, 257, 256, False)[0]


def test_sequences_without_a_mask():
    """2^22 workgroups of 1,024 threads would put masks' visible keys in order."""
    assert taken(1 << 22, 1, 1, 1, 129, False) == (True, True)
    assert taken(1 << 22, 1, 1, 1, 129, True) == (True, False)
    assert taken((1 << 22) - 1, 1, 1, 1, 129, True) == (True, True)
