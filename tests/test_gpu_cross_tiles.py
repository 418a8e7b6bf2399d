"""Cross attention of many rows on the GPU, against its definition in 64 bits: calls
whose groups of 32 rows pass the chip's compute units, which run in tiles of 256 rows --
over keys that all lie in LDS (up to 256) or pass through it, tiles of few heads over
many keys shared between workgroups.  Tolerances: test_gpu_cross_attn.py's."""
import math

import pytest
import torch

from paper_2609_35110_amd import sol
from test_gpu_cross_attn import check, inputs, near, reference, visible

pytestmark = pytest.mark.gpu
D = 128
# whole tiles of rows, their last ones of one row and more; shared tiles (the last two)
RING = [(1, 35, 35, 257, 300), (2, 16, 4, 300, 513), (3, 7, 7, 450, 290), (5, 8, 8, 256, 257), (1, 36, 36, 256, 1100), (1, 40, 8, 230, 1500)]
BRIEF = [(1, 35, 35, 257, M) for M in (1, 2, 31, 32, 33, 64, 65, 96, 128, 129, 256)] + \
    [(2, 16, 4, 300, 200), (40, 4, 4, 65, 77), (3, 7, 7, 450, 160)]
FEW_OF_EACH = [(1, 36, 36, 256, 1100), (2, 16, 4, 300, 513), (2, 16, 4, 300, 200), (3, 7, 7, 450, 77)]


def some_mask(B, M, share, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.rand(B, M, generator=g) < share).to(torch.uint8) * torch.randint(1, 256, (B, M), generator=g).to(torch.uint8)


def spread(n, B):
    """Lengths past n and below 0 among them."""
    return torch.tensor([9999999, n // 2, 1, -3, n][:B], dtype=torch.int32)


@pytest.mark.parametrize("B,H,Hk,N,M", RING + BRIEF)
def test_against_definition(B, H, Hk, N, M):
    check(inputs(B, H, Hk, N, M, seed=N + M))


@pytest.mark.parametrize("share", [0.0, 0.05, 0.5, 1.0])
@pytest.mark.parametrize("B,H,Hk,N,M", FEW_OF_EACH)
def test_masked_keys(B, H, Hk, N, M, share):
    x = inputs(B, H, Hk, N, M, seed=M)
    mask = some_mask(B, M, share, M)
    check(x, key_mask=mask)
    check(x, key_mask=mask.bool(), kv_lens=spread(M, B), q_lens=spread(N, B).flip(0))


@pytest.mark.parametrize("H,Hk,N,M", [(4, 2, 700, 300), (4, 2, 700, 200), (8, 8, 257, 1100), (6, 1, 520, 31)])
def test_ragged_batch(H, Hk, N, M):
    x = inputs(5, H, Hk, N, M, seed=4)
    check(x, q_lens=torch.tensor([N, 1, 0, 257, 256], dtype=torch.int32), kv_lens=torch.tensor([1, M, 77, 0, M - 1], dtype=torch.int32))
    check(x, q_lens=spread(N, 5), kv_lens=spread(M, 5).flip(0))
    check(x, q_lens=torch.zeros(5, dtype=torch.int32))


def test_more_sequences_than_lengths_are_added_up_for():
    """Past 1,024 sequences every one counts as a whole one."""
    x = inputs(1100, 1, 1, 40, 20, seed=6)
    g = torch.Generator().manual_seed(6)
    ql, kl = (torch.randint(0, n + 1, (1100,), generator=g, dtype=torch.int32) for n in (40, 20))
    check(x, q_lens=ql, kv_lens=kl, key_mask=some_mask(1100, 20, 0.7, 6))
    x = inputs(1100, 1, 1, 9, 260, seed=6)
    check(x, q_lens=ql.clamp(max=9), kv_lens=kl * 13, key_mask=some_mask(1100, 260, 0.7, 6))


@pytest.mark.parametrize("H,N,M", [(34, 256, 300), (34, 256, 200), (36, 256, 1100)])
def test_one_visible_key_anywhere(H, N, M):
    x = inputs(1, H, 1, N, M, seed=2)
    y = {n: t.cuda() for n, t in x.items()}
    for at in (0, 31, 32, 127, 128, M - 1):
        mask = torch.zeros(1, M, dtype=torch.uint8, device="cuda")
        mask[0, at] = 1
        out, left, lse = sol.cross_attn_fwd(y["q"], y["k"], y["v"], key_mask=mask, training=True)
        assert torch.equal(out, y["v"][:, :, at:at + 1].expand_as(out)) and not left.any()
        dq, dk, dv = sol.cross_attn_bwd(y["do"], y["q"], y["k"], y["v"], out, left, lse, key_mask=mask)
        hidden = (mask[0] == 0).cpu()
        assert not dk[0, 0, hidden.cuda()].any() and not dv[0, 0, hidden.cuda()].any()
        near(dv, torch.where(hidden[:, None], 0.0, x["do"].double().sum((1, 2))[:, None, None]))


@pytest.mark.parametrize("H,N,M", [(18, 300, 300), (18, 300, 150), (20, 256, 1300)])
def test_what_is_hidden_is_not_read(H, N, M):
    B = 2
    x = inputs(B, H, H // 2, N, M, seed=3)
    mask = some_mask(B, M, 0.6, 3)
    kv, ql = torch.tensor([M - 7, 64], dtype=torch.int32), torch.tensor([N, N - 9], dtype=torch.int32)
    want = check(x, key_mask=mask, kv_lens=kv, q_lens=ql)
    _, rows, keys = visible(x, ql, kv, mask)
    g = torch.Generator().manual_seed(4)
    junk = torch.tensor([math.nan, math.inf, -math.inf, 3e38])[torch.randint(0, 4, (B, 1, max(M, N), 1), generator=g)].bfloat16()
    y = {n: torch.where(keys, x[n], junk[:, :, :M]).cuda() for n in ("k", "v")}
    y.update({n: torch.where(rows, x[n], junk[:, :, :N]).cuda() for n in ("q", "do")})
    dm = dict(key_mask=mask.cuda(), kv_lens=kv.cuda(), q_lens=ql.cuda())
    out, left, lse = sol.cross_attn_fwd(y["q"], y["k"], y["v"], out=torch.full_like(want[0], 7.0), training=True, **dm)
    assert torch.equal(out, want[0])
    got = sol.cross_attn_bwd(y["do"], y["q"], y["k"], y["v"], out, left, lse, **dm)
    assert all(torch.equal(a, b) for a, b in zip(got, want[1]))


@pytest.mark.parametrize("H,N,M", [(34, 256, 400), (34, 256, 250), (40, 230, 1500)])
def test_peaked_rows(H, N, M):
    """1 % of the keys times 8: scores of 90 and more, maxima that come late."""
    check(inputs(1, H, H // 2, N, M, seed=5, boost=True))


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("H,N,M", [(34, 256, 400), (34, 256, 250), (40, 230, 1500)])
def test_maxima_far_above_the_first_keys(H, N, M, masked):
    """Keys late in the sequence whose scores are hundreds above the first tile's, for some heads alone."""
    x = inputs(1, H, H, N, M, seed=7)
    x["k"][:, ::3, M - 50:M - 47] *= 64
    x["k"][:, 1::3, M // 2] *= 24
    check(x, **(dict(key_mask=some_mask(1, M, 0.7, 7) | (torch.arange(M) >= M - 60).to(torch.uint8)) if masked else {}))


@pytest.mark.parametrize("H,N,M", [(34, 256, 300), (34, 256, 100), (40, 230, 1500)])
def test_large_values_under_late_maxima(H, N, M):
    """Values of 2^90 whose products with P of 2^60 would leave fp32: scores are held to the rows' own maxima."""
    x = inputs(1, H, 1, N, M, seed=8)
    x["v"] = (x["v"].float() * 2.0 ** 90).bfloat16()
    x["k"][:, :, M - 30] *= 24
    ref = reference(x)[0]
    y = {n: t.cuda() for n, t in x.items()}
    near(sol.cross_attn_fwd(y["q"], y["k"], y["v"]).double() * 2.0 ** -90, ref * 2.0 ** -90)


@pytest.mark.parametrize("M", [300, 100])
@pytest.mark.parametrize("scale", [1e-30, 0.01, 1.0])
def test_scales(scale, M):
    check(inputs(1, 34, 17, 256, M, seed=9), scale=scale)


@pytest.mark.parametrize("M", [300, 100])
@pytest.mark.parametrize("order", [(0, 2, 1, 3), (1, 0, 2, 3), (2, 0, 1, 3)])
def test_strides(order, M):
    back = [order.index(i) for i in range(4)]
    place = lambda t: t.permute(*order).contiguous().permute(*back)  # noqa: E731
    x = inputs(2, 16, 4, 300, M, seed=10)
    check(x, place=place, key_mask=some_mask(2, M, 0.8, 1))
    wide = lambda t: torch.cat([t, torch.full_like(t, float("nan"))], -1)[..., :D]  # noqa: E731
    check(x, place=wide, kv_lens=torch.tensor([100, 33], dtype=torch.int32))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("name", ["q", "k", "v", "do"])
@pytest.mark.parametrize("M", [500, 150, 100])
def test_a_value_that_is_not_finite_stays_in_its_sequence_and_heads(name, bad, M):
    """One such value in a sequence's last token, whose tile others follow."""
    x = {n: t.cuda() for n, t in inputs(2, 16, 8, 700, M, seed=1).items()}

    def run():
        args = (x["q"], x["k"], x["v"])
        fwd = sol.cross_attn_fwd(*args, training=True)
        return (*fwd, *sol.cross_attn_bwd(x["do"], *args, *fwd))

    want = run()
    x[name][0, 2, -1, 5] = bad
    got = run()
    key_head = 1 if name in ("q", "do") else 2  # of 8, which two heads share
    assert not torch.isfinite(got[3][0, [2 * key_head, 2 * key_head + 1]].float()).all()
    for a, b in zip(want, got):
        per = a.shape[1] // 8
        others = [h for h in range(a.shape[1]) if h // per != key_head]
        assert torch.equal(b[1], a[1]) and torch.equal(b[0, others], a[0, others])
