"""The C ABI of the norm and rotation at given positions and of cross attention
without a GPU: every refusal happens on the host, before any HIP call (the pointers
here are never read)."""
import os

import pytest

from paper_2609_35110_amd import sol
from test_ops_abi import S, at, refused


@pytest.fixture(scope="module", autouse=True)
def L():
    if not os.path.exists(sol.LIB_PATH):
        from paper_2609_35110_amd import build
        build.build()
    return sol.lib()


nan, inf = float("nan"), float("inf")
BIG = 1 << 40
ROPE = dict(q=at(1), q_st=None, k=at(2), k_st=None, qg=at(3), kg=at(4), eps=1e-6, pos=at(5), pos_sb=300, tab=at(6), T=9,
            Hl=5, Wl=7, dt=32, dh=48, dw=48, lens=None, B=2, H=4, Hk=2, N=100, D=128)
ROPE_COMMON = [
    (dict(B=0), -1, ">= 1"),
    (dict(H=0), -1, ">= 1"),
    (dict(Hk=-1), -1, ">= 0"),
    (dict(N=0), -1, ">= 1"),
    (dict(D=64), -2, "head dim"),
    (dict(N=(1 << 23) + 1), -2, "exceeds"),
    (dict(B=32, N=1 << 23), -2, "B*N too large"),
    (dict(B=(1 << 28) - 15, N=1), -2, "B*N too large"),
    (dict(H=1 << 16), -2, "H + Hk too large"),
    (dict(H=(1 << 16) - 2), -2, "H + Hk too large"),
    (dict(H=2147483647, Hk=2147483647), -2, "H + Hk too large"),
    (dict(eps=-1e-9), -1, "eps"),
    (dict(eps=nan), -1, "eps"),
    (dict(eps=inf), -1, "eps"),
    (dict(qg=at(3) + 4), -1, "q_gamma and k_gamma"),
    (dict(kg=at(4) + 8), -1, "q_gamma and k_gamma"),
    (dict(Hk=0), -1, "k_gamma without k"),
    (dict(dt=-8), -1, "split"),
    (dict(dh=44), -1, "split"),
    (dict(dw=56), -1, "split"),
    (dict(dt=2147483640, dh=2147483640), -1, "split"),
    (dict(T=-1), -1, "T, Hl, Wl"),
    (dict(T=1 << 24, Hl=1 << 24), -2, "too large together"),
    (dict(pos=at(5) + 2), -1, "pos must be 4-byte"),
    (dict(lens=at(7) + 1), -1, "lens must be 4-byte"),
    (dict(tab=None), -1, "rope_tab must not be NULL"),
    (dict(tab=at(6) + 8), -1, "rope_tab must be 16-byte"),
    (dict(pos_sb=-1), -1, "pos_stride_b"),
    (dict(pos_sb=299), -1, "pos_stride_b"),
    (dict(pos_sb=BIG + 1), -1, "pos_stride_b"),
]


def rope(**kw):
    a = dict(ROPE, yq=at(11), yq_st=None, yk=at(12), yk_st=None)
    a.update(kw)
    return sol.sol_qk_norm_rope(a["q"], a["q_st"], a["k"], a["k_st"], a["yq"], a["yq_st"], a["yk"], a["yk_st"], a["qg"],
                                a["kg"], a["eps"], a["pos"], a["pos_sb"], a["tab"], a["T"], a["Hl"], a["Wl"], a["dt"],
                                a["dh"], a["dw"], a["lens"], a["B"], a["H"], a["Hk"], a["N"], a["D"], None)


@pytest.mark.parametrize("kw,status,fragment", ROPE_COMMON + [
    (dict(q=None), -1, "q must not be NULL"),
    (dict(q=at(1) + 8), -1, "q must be 16-byte"),
    (dict(k=None), -1, "k must not be NULL"),
    (dict(yq=None), -1, "q_out must not be NULL"),
    (dict(yk=None), -1, "k_out must not be NULL"),
    (dict(q_st=S(4 * 100 * 128, 100 * 128, 129)), -1, "q strides"),
    (dict(k_st=S(-8, 100 * 128, 128)), -1, "k strides"),
    (dict(k_st=S(0, 0, (1 << 24) + 8)), -2, "between tokens"),
    (dict(yq_st=S(4 * 100 * 128, 0, 128)), -1, "rows of q_out overlap"),
    (dict(yk_st=S(100 * 128, 100 * 128, 128)), -1, "rows of k_out overlap"),
    (dict(yq=at(1) + 256), -1, "q_out overlaps q"),                          # another row's place
    (dict(yq=at(1), yq_st=S(4 * 100 * 128, 128, 512)), -1, "q_out overlaps q"),  # in place, in another order
    (dict(yk=at(1)), -1, "k_out overlaps q"),
    (dict(yq=at(2)), -1, "q_out overlaps k"),
    (dict(yk=at(11)), -1, "k_out overlaps q_out"),
    (dict(yq=at(3) - 256), -1, "q_out overlaps q_gamma"),
    (dict(yq=at(5) - 1024), -1, "q_out overlaps pos"),
    (dict(yk=at(6)), -1, "k_out overlaps rope_tab"),
    (dict(yk=at(7), lens=at(7) + 64), -1, "k_out overlaps lens"),
])
def test_norm_rope_refusals(kw, status, fragment):
    refused(status, fragment, rope(**kw))


def rope_bwd(**kw):
    a = dict(ROPE, gq=at(13), gk=at(14), dq=at(11), dq_st=None, dk=at(12), dk_st=None, dqg=at(15), dkg=at(16), ws=at(17),
             ws_bytes=1 << 25)
    a.update(kw)
    return sol.sol_qk_norm_rope_bwd(a["gq"], None, a["gk"], None, a["q"], a["q_st"], a["k"], a["k_st"], a["dq"], a["dq_st"],
                                    a["dk"], a["dk_st"], a["qg"], a["kg"], a["dqg"], a["dkg"], a["eps"], a["pos"],
                                    a["pos_sb"], a["tab"], a["T"], a["Hl"], a["Wl"], a["dt"], a["dh"], a["dw"], a["lens"],
                                    a["B"], a["H"], a["Hk"], a["N"], a["D"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status,fragment", ROPE_COMMON + [
    (dict(q=None), -1, "q must not be NULL"),          # (there is a gamma)
    (dict(k=None), -1, "k must not be NULL"),
    (dict(gq=None), -1, "dq_out must not be NULL"),
    (dict(gk=at(14) + 4), -1, "dk_out must be 16-byte"),
    (dict(dq=None), -1, "dq must not be NULL"),
    (dict(dk=None), -1, "dk must not be NULL"),
    (dict(dk_st=S(2 * 100 * 128, 0, 128)), -1, "rows of dk overlap"),
    (dict(qg=None), -1, "a gradient of weights"),
    (dict(kg=None), -1, "a gradient of weights"),
    (dict(dqg=at(15) + 2), -1, "dq_gamma must be 4-byte"),
    (dict(dkg=at(15) + 256), -1, "dk_gamma overlaps dq_gamma"),
    (dict(dqg=at(3)), -1, "dq_gamma overlaps q_gamma"),
    (dict(dq=at(1)), -1, "dq overlaps q"),             # (in place of dq_out alone)
    (dict(dq=at(14)), -1, "dq overlaps dk_out"),
    (dict(dk=at(11)), -1, "dk overlaps dq"),
    (dict(ws=None), -1, "workspace is NULL"),
    (dict(ws=at(17) + 8), -1, "workspace must be 16-byte"),
    (dict(ws_bytes=1000), -1, "workspace needs"),
    (dict(ws=at(2)), -1, "workspace overlaps k"),
    (dict(ws=at(15)), -1, "workspace overlaps dq_gamma"),
])
def test_norm_rope_bwd_refusals(kw, status, fragment):
    refused(status, fragment, rope_bwd(**kw))


def test_norm_rope_workspaces():
    # two sums of 128 floats a workgroup: tokens in sixteens, up to 2,048 workgroups in rounds of them
    assert sol.sol_qk_norm_rope_bwd_workspace_bytes(1, 1, 0, 1, 128) == 1024
    assert sol.sol_qk_norm_rope_bwd_workspace_bytes(1, 1, 1, 17, 128) == 4 * 1024
    for sizes in ((1, 24, 24, 1, 128), (3, 7, 2, 1000, 128), (1, 24, 24, 1 << 20, 128), (1, 60000, 5000, 1, 128)):
        need = sol.sol_qk_norm_rope_bwd_workspace_bytes(*sizes)
        assert need and need % 1024 == 0 and need <= 1024 * max(4096, sizes[1] + sizes[2])
    for bad in ((0, 1, 1, 1, 128), (1, 1, -1, 1, 128), (1, 1, 1, 1, 64), (1, 1 << 16, 0, 1, 128), (1 << 28, 1, 0, 1, 128)):
        assert sol.sol_qk_norm_rope_bwd_workspace_bytes(*bad) == 0


CROSS = dict(q=at(1), k=at(2), k_st=None, v=at(3), v_st=None, out=at(4), out_st=None, left=at(5), lse=at(6), q_lens=None,
             kv_lens=None, mask=None, B=2, H=4, Hk=2, N=100, M=120, D=128, scale=0.1)
CROSS_COMMON = [
    (dict(B=0), -1, ">= 1"),
    (dict(H=0), -1, ">= 1"),
    (dict(Hk=0), -1, ">= 1"),
    (dict(N=0), -1, ">= 1"),
    (dict(M=0), -1, ">= 1"),
    (dict(Hk=3), -1, "multiple"),
    (dict(Hk=8), -1, "multiple"),
    (dict(D=256), -2, "head dim"),
    (dict(N=(1 << 23) + 1), -2, "exceeds"),
    (dict(M=(1 << 23) + 1), -2, "exceeds"),
    (dict(B=1 << 12, H=1 << 12), -2, "too large"),
    (dict(B=1 << 10, N=1 << 20), -2, "too large"),
    (dict(B=1 << 10, M=1 << 20), -2, "too large"),
    (dict(scale=0.0), -1, "scale"),
    (dict(scale=-0.1), -1, "scale"),
    (dict(scale=nan), -1, "scale"),
    (dict(scale=inf), -1, "scale"),
    (dict(scale=1e-31), -1, "scale must be 1e-30"),
    (dict(scale=2e8), -1, "scale must be 1e-30"),
    (dict(q_lens=at(7) + 1), -1, "q_lens must be 4-byte"),
    (dict(kv_lens=at(7) + 2), -1, "kv_lens must be 4-byte"),
    (dict(q=None), -1, "q must not be NULL"),
    (dict(q=at(1) + 2), -1, "q must be 16-byte"),
    (dict(k=at(2) + 8), -1, "k must be 16-byte"),
    (dict(v=None), -1, "v must not be NULL"),
    (dict(out=None), -1, "out must not be NULL"),
    (dict(k_st=S(0, 0, 4)), -1, "k strides"),
    (dict(v_st=S(0, -8, 128)), -1, "v strides"),
    (dict(v_st=S(0, 0, (1 << 24) + 8)), -2, "between tokens"),
    (dict(left=at(5) + 8), -1, "out_left must be 16-byte"),
    (dict(lse=at(6) + 2), -1, "lse must be 4-byte"),
]


def cross_fwd(**kw):
    a = dict(CROSS, ws=None, ws_bytes=0)
    a.update(kw)
    return sol.sol_cross_attn_fwd(a["q"], None, a["k"], a["k_st"], a["v"], a["v_st"], a["out"], a["out_st"], a["left"],
                                  a["lse"], a["q_lens"], a["kv_lens"], a["mask"], a["B"], a["H"], a["Hk"], a["N"], a["M"],
                                  a["D"], a["scale"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status,fragment", CROSS_COMMON + [
    (dict(left=None), -1, "given together"),
    (dict(lse=None), -1, "given together"),
    (dict(out=at(1)), -1, "out overlaps q"),
    (dict(out=at(3)), -1, "out overlaps v"),
    (dict(out_st=S(0, 100 * 128, 128)), -1, "rows of out overlap"),
    (dict(left=at(4)), -1, "out_left overlaps out"),
    (dict(left=at(2)), -1, "out_left overlaps k"),
    (dict(lse=at(5) + 64), -1, "lse overlaps out_left"),
    (dict(q_lens=at(4) + 64), -1, "out overlaps q_lens"),
    (dict(mask=at(4) + 65, N=1), -1, "out overlaps key_mask"),
    (dict(mask=at(7) + 1, N=2000, M=300), -1, "workspace is NULL"),  # (the visible keys' order)
    (dict(N=1, M=30000), -1, "workspace is NULL"),                # pieces of the keys
    (dict(N=1, M=30000, ws=at(9) + 8, ws_bytes=1 << 30), -1, "workspace must be 16-byte"),
    (dict(N=1, M=30000, ws=at(9), ws_bytes=64), -1, "workspace needs"),
    (dict(N=1, M=30000, ws=at(3), ws_bytes=1 << 30), -1, "workspace overlaps"),
    (dict(B=1 << 20, H=2, Hk=1, N=65, M=300, q=at(1), out=1 << 46, k=1 << 47, v=1 << 48, left=None, lse=None), -2,
     "too large together"),
])
def test_cross_fwd_refusals(kw, status, fragment):
    refused(status, fragment, cross_fwd(**kw))


def cross_bwd(**kw):
    a = dict(CROSS, dout=at(10), dq=at(11), dk=at(12), dv=at(13), dv_st=None, ws=at(14), ws_bytes=1 << 26)
    a.update(kw)
    return sol.sol_cross_attn_bwd(a["dout"], None, a["q"], None, a["k"], a["k_st"], a["v"], a["v_st"], a["out"], a["out_st"],
                                  a["left"], a["lse"], a["dq"], None, a["dk"], None, a["dv"], a["dv_st"], a["q_lens"],
                                  a["kv_lens"], a["mask"], a["B"], a["H"], a["Hk"], a["N"], a["M"], a["D"], a["scale"],
                                  a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status,fragment", CROSS_COMMON + [
    (dict(left=None), -1, "out_left must not be NULL"),
    (dict(lse=None), -1, "lse must not be NULL"),
    (dict(dout=None), -1, "dout must not be NULL"),
    (dict(dq=at(11) + 8), -1, "dq must be 16-byte"),
    (dict(dk=None), -1, "dk must not be NULL"),
    (dict(dq=at(10)), -1, "dq overlaps dout"),
    (dict(dk=at(2)), -1, "dk overlaps k"),
    (dict(dv=at(12)), -1, "dv overlaps dk"),
    (dict(dq=at(4)), -1, "dq overlaps out"),
    (dict(dv=at(5)), -1, "dv overlaps out_left"),
    (dict(dk=at(6)), -1, "dk overlaps lse"),
    (dict(dv=at(7), mask=at(7) + 64), -1, "dv overlaps key_mask"),
    (dict(dv_st=S(2 * 120 * 128, 0, 128)), -1, "rows of dv overlap"),
    (dict(dv_st=S(0, 120 * 128, 128)), -1, "rows of dv overlap"),
    (dict(ws=None), -1, "workspace is NULL"),
    (dict(ws=at(14) + 4), -1, "workspace must be 16-byte"),
    (dict(ws_bytes=100), -1, "workspace needs"),
    (dict(ws=at(2)), -1, "workspace overlaps k"),
    (dict(ws=at(6)), -1, "workspace overlaps lse"),
    (dict(B=1 << 20, H=4, N=65, M=300), -2, "too large together"),
])
def test_cross_bwd_refusals(kw, status, fragment):
    refused(status, fragment, cross_bwd(**kw))


def test_cross_workspaces():
    fwd, bwd = sol.sol_cross_attn_fwd_workspace_bytes, sol.sol_cross_attn_bwd_workspace_bytes
    assert fwd(1, 24, 24, 1, 512, 128, 0) == 0          # few rows, one piece
    assert fwd(1, 24, 24, 1, 512, 128, 1) == 0          # (which reads the mask itself)
    assert fwd(1, 1, 1, 1, 30000, 128, 0) > 0           # pieces
    assert fwd(4, 24, 24, 8192, 512, 128, 0) == 0       # whole tiles
    assert fwd(4, 24, 24, 8192, 256, 128, 1) == 0       # all keys at once
    # the visible keys' lists and how many there are, in 256 bytes
    for B, M in ((1, 257), (3, 263), (2, 397), (5, 512)):
        assert fwd(B, 16, 16, 4096, M, 128, 1) - fwd(B, 16, 16, 4096, M, 128, 0) == (4 * (B * M + B) + 255) // 256 * 256
        assert bwd(B, 16, 16, 4096, M, 128, 1) - bwd(B, 16, 16, 4096, M, 128, 0) == (4 * (B * M + B) + 255) // 256 * 256
    assert bwd(1, 24, 24, 32, 77, 128, 1) == 0          # a key head's rows in one workgroup
    assert bwd(1, 24, 24, 4096, 77, 128, 1) == 24 * 10 * 2 * 128 * 128 * 4  # in ten, joined
    for bad in ((0, 1, 1, 1, 1, 128, 0), (1, 1, 1, 1, 0, 128, 0), (1, 3, 2, 1, 1, 128, 0), (1, 1, 1, 1, 1, 64, 0),
                (1 << 12, 1 << 11, 1, 1, 1, 128, 0), (1 << 10, 1, 1, 1 << 22, 1, 128, 0)):
        assert fwd(*bad) == 0 and bwd(*bad) == 0
