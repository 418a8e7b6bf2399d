"""Cross attention on the GPU, against its definition in 64 bits (plain torch on the
CPU), through the torch binding.

Tolerances, as the differential attention's: a bf16 result is rounded once, P (and,
backwards, dS) once before a product: each a relative error of at most 2^-8 per term,
1.7e-3 in the mean square over a binade; three of them give 3e-3 of a result's norm:
TOL_BF16 = 5e-3.  The worst single value: 6 standard deviations of 2 x 1.7e-3 of the
rms plus its own rounding: MAX_BF16 = 3e-2 of the larger of rms and value, the rms being
that of its row of 128 where that is the larger one (a row's 128 sums have the same
weights).  delta = dout . out is found from the output of rounded P, divided by the sum
of the rounded ones: off by sum_j e_j P_j (X_j - delta), e_j the roundings, so by at most
6 standard deviations, 6 x 1.7e-3 x sqrt(sum P^2 (X - delta)^2); and from an output kept
in two bf16 parts: 2^-16 sum |dout| |out|.  It is the same for all of a row's keys; what
it adds to dq and dk is computed beside the reference and allowed on top.  lse: scores
are exact products summed in fp32 over 128 terms, 128 x 2^-24 x |score| at most and the
final log: 1e-5 x the largest |score| + 1e-6."""
import math

import pytest
import torch

from paper_2609_35110_amd import sol

pytestmark = pytest.mark.gpu
D = 128
TOL_BF16, MAX_BF16 = 5e-3, 3e-2


def inputs(B, H, Hk, N, M, seed=0, boost=False):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g).bfloat16()  # noqa: E731
    x = {"q": r(B, H, N, D), "k": r(B, Hk, M, D), "v": r(B, Hk, M, D), "do": r(B, H, N, D)}
    if boost:
        x["k"][:, :, torch.randperm(M, generator=g)[: max(1, M // 100)]] *= 8
    return x


def visible(x, q_lens=None, kv_lens=None, key_mask=None):
    """[B, 1, N, M]: which keys a row sees, and [B, 1, N, 1]: which rows are the sequences'."""
    B, _, N, _ = x["q"].shape
    M = x["k"].shape[2]
    ql = torch.full((B,), N) if q_lens is None else q_lens.clamp(0, N)
    kl = torch.full((B,), M) if kv_lens is None else kv_lens.clamp(0, M)
    keys = torch.arange(M) < kl[:, None]
    if key_mask is not None:
        keys = keys & (key_mask != 0)
    rows = torch.arange(N) < ql[:, None]
    return (keys[:, None, None, :] & rows[:, None, :, None]), rows[:, None, :, None], keys[:, None, :, None]


def maps(x, scale, **masks):
    """P [B, H, N, M] in 64 bits, the log sums, and the operands with what is not seen at 0."""
    H, Hk = x["q"].shape[1], x["k"].shape[1]
    seen, rows, keys = visible(x, **masks)
    wide = lambda t: torch.where(keys, t.double(), 0.0).repeat_interleave(H // Hk, 1)  # noqa: E731
    q, k, v = torch.where(rows, x["q"].double(), 0.0), wide(x["k"]), wide(x["v"])
    s = torch.where(seen, q @ k.transpose(-1, -2) * scale, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse.isinf(), 0.0, lse)[..., None])
    return p, lse, q, k, v, torch.where(rows, x["do"].double(), 0.0), rows, s


def reference(x, scale=D ** -0.5, **masks):
    """out, (dq, dk, dv), lse, the allowances of dq and dk, and the scores."""
    B, H, N, _ = x["q"].shape
    Hk, M = x["k"].shape[1], x["k"].shape[2]
    p, lse, q, k, v, do, _, s = maps(x, scale, **masks)
    out = p @ v
    X = do @ v.transpose(-1, -2)
    delta = (out * do).sum(-1, keepdim=True)
    dS = p * (X - delta) * scale
    heads = lambda t: t.reshape(B, Hk, H // Hk, M, D).sum(2)  # noqa: E731
    err = 6 * 1.7e-3 * (p * (X - delta)).norm(dim=-1, keepdim=True) + 2.0 ** -16 * (do.abs() * out.abs()).sum(-1, keepdim=True)
    err = err * scale
    aq, ak = (err * (p @ k).abs()).norm(), heads((p * err).transpose(-1, -2) @ q.abs()).norm()
    return out, (dS @ k, heads(dS.transpose(-1, -2) @ q), heads(p.transpose(-1, -2) @ do)), lse, (aq, ak, 0.0), s


def near(x, ref, extra=0.0):
    x, ref = x.double().cpu(), ref.double()
    assert x.shape == ref.shape and torch.isfinite(x).all()
    norm, d = ref.norm(), (x - ref).abs()
    assert d.norm() <= TOL_BF16 * norm + extra
    rms = torch.maximum(norm / math.sqrt(ref.numel()), ref.norm(dim=-1, keepdim=True) / math.sqrt(ref.shape[-1]))
    assert (d <= MAX_BF16 * torch.maximum(rms, ref.abs()) + extra).all()


def check(x, scale=None, place=lambda t: t, **masks):
    """Both directions; place: how a tensor lies in device memory (a view of its values)."""
    ref, grads, lse, extra, s = reference(x, scale or D ** -0.5, **masks)
    y = {n: place(t.cuda()) for n, t in x.items()}
    dm = {n: t.cuda() if t is not None else None for n, t in masks.items()}
    rows = visible(x, **masks)[1]
    inside = rows.expand(ref.shape)
    args = (y["q"], y["k"], y["v"])
    start = torch.full(ref.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    out, left, l = sol.cross_attn_fwd(*args, scale=scale, out=place(start.clone()), training=True, **dm)
    assert (out.cpu()[~inside] == 7.0).all()
    near(torch.where(rows, out.cpu().double(), 0.0), ref)
    l, some, valid = l.cpu(), torch.isfinite(lse), rows[..., 0].expand(lse.shape)
    assert torch.equal(torch.isfinite(l)[valid], some[valid]) and (l[valid & ~some] == -math.inf).all()
    assert (out.cpu()[(valid & ~some)] == 0).all()
    if some.any():
        most = s[torch.isfinite(s)].abs().max()
        assert (l.double() - lse)[some & valid].abs().max() <= 1e-5 * most + 1e-6
    alone = sol.cross_attn_fwd(*args, scale=scale, out=place(start.clone()), **dm)
    assert torch.equal(alone, out)
    # the output for training in two parts: as exact as the probabilities' rounding leaves it
    near(torch.where(rows, out.cpu().double() + left.cpu().double(), 0.0), ref)
    got = sol.cross_attn_bwd(y["do"], *args, out, left, torch.as_tensor(l).cuda(), scale=scale, **dm)
    for a, b, e in zip(got, grads, extra):
        near(a, b, e)
    again = sol.cross_attn_bwd(y["do"], *args, out, left, torch.as_tensor(l).cuda(), scale=scale, **dm)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    return out, got


SHAPES = [(1, 1, 1, 1, 1), (1, 1, 1, 1, 2), (2, 2, 1, 3, 70), (1, 2, 2, 64, 64), (1, 4, 2, 65, 127), (1, 1, 1, 128, 129),
          (2, 3, 3, 130, 31), (1, 2, 1, 257, 300), (1, 2, 2, 500, 1), (1, 2, 1, 300, 1100), (2, 2, 2, 511, 33),
          (1, 6, 2, 256, 32), (1, 1, 1, 700, 512)]


@pytest.mark.parametrize("B,H,Hk,N,M", SHAPES)
def test_against_definition(B, H, Hk, N, M):
    check(inputs(B, H, Hk, N, M, seed=N + M))


@pytest.mark.parametrize("share", [0.0, 0.05, 0.5, 1.0])
@pytest.mark.parametrize("B,H,Hk,N,M", [(2, 2, 1, 1, 1), (3, 4, 2, 5, 333), (2, 2, 2, 300, 65), (3, 3, 1, 700, 200), (2, 1, 1, 260, 1030)])
def test_masked_keys(B, H, Hk, N, M, share):
    """From none visible (rows without keys, gradients of 0) to all."""
    g = torch.Generator().manual_seed(M)
    mask = (torch.rand(B, M, generator=g) < share).to(torch.uint8) * torch.randint(1, 256, (B, M), generator=g).to(torch.uint8)
    x = inputs(B, H, Hk, N, M, seed=M)
    check(x, key_mask=mask)
    check(x, key_mask=mask.bool(), kv_lens=torch.tensor([M, M // 2, 0][:B], dtype=torch.int32))


def test_one_visible_key_anywhere():
    """A single key, at the place of each of a tile's corners: out is its value, dq and dk are 0 but for roundings."""
    x = inputs(1, 1, 1, 300, 200, seed=2)
    for at in (0, 31, 32, 127, 128, 199):
        mask = torch.zeros(1, 200, dtype=torch.uint8)
        mask[0, at] = 1
        y = {n: t.cuda() for n, t in x.items()}
        out, left, lse = sol.cross_attn_fwd(y["q"], y["k"], y["v"], key_mask=mask.cuda(), training=True)
        assert torch.equal(out, y["v"][:, :, at:at + 1].expand_as(out))
        dq, dk, dv = sol.cross_attn_bwd(y["do"], y["q"], y["k"], y["v"], out, left, lse, key_mask=mask.cuda())
        hidden = mask[0] == 0
        assert (dk[0, 0, hidden.cuda()] == 0).all() and (dv[0, 0, hidden.cuda()] == 0).all()
        near(dv, torch.where(hidden[:, None], 0.0, x["do"].double().sum(2, keepdim=True)))
        # X - delta is the difference of two sums of 128 products in fp32, each within 128 x 2^-24 of the terms' sizes
        size = (x["do"].double().abs() * x["v"][:, :, at:at + 1].double().abs()).sum(-1, keepdim=True) * 2 * 128 * 2.0 ** -24
        assert (dq.cpu().double().abs() <= D ** -0.5 * size * x["k"][:, :, at:at + 1].double().abs() * 1.01).all()


@pytest.mark.parametrize("N", [3, 400])
def test_what_is_hidden_is_not_read(N):
    """NaN and infinities in hidden keys, behind sequences, and in rows behind them."""
    B, H, Hk, M = 2, 2, 1, 150
    g = torch.Generator().manual_seed(3)
    x = inputs(B, H, Hk, N, M, seed=3)
    mask = torch.rand(B, M, generator=g) < 0.6
    kv = torch.tensor([M - 7, 64], dtype=torch.int32)
    ql = torch.tensor([N, max(1, N - 9)], dtype=torch.int32)
    want = check(x, key_mask=mask, kv_lens=kv, q_lens=ql)
    seen, rows, keys = visible(x, ql, kv, mask)
    bad = {n: t.clone() for n, t in x.items()}
    junk = torch.tensor([math.nan, math.inf, -math.inf, 3e38])[torch.randint(0, 4, (B, 1, max(M, N), 1), generator=g)].bfloat16()
    for n in ("k", "v"):
        bad[n] = torch.where(keys, bad[n], junk[:, :, :M])
    for n in ("q", "do"):
        bad[n] = torch.where(rows, bad[n], junk[:, :, :N])
    y = {n: t.cuda() for n, t in bad.items()}
    dm = dict(key_mask=mask.cuda(), kv_lens=kv.cuda(), q_lens=ql.cuda())
    out, left, lse = sol.cross_attn_fwd(y["q"], y["k"], y["v"], out=torch.full_like(want[0], 7.0), training=True, **dm)
    assert torch.equal(out, want[0])
    got = sol.cross_attn_bwd(y["do"], y["q"], y["k"], y["v"], out, left, lse, **dm)
    assert all(torch.equal(a, b) for a, b in zip(got, want[1]))


@pytest.mark.parametrize("B,H,Hk,N,M", [(1, 1, 1, 1, 5000), (1, 6, 2, 1, 2100), (2, 4, 1, 8, 1100), (1, 8, 1, 4, 1024),
                                        (1, 2, 1, 17, 2048), (2, 36, 1, 1, 2100), (32, 4, 4, 1, 300), (1, 40, 1, 2, 1300)])
def test_few_rows(B, H, Hk, N, M):
    """Single tokens and drafted ones over an encoder's states: keys are split and joined."""
    x = inputs(B, H, Hk, N, M, seed=M)
    check(x)
    kv = torch.arange(B, dtype=torch.int32) * 99 % M
    g = torch.Generator().manual_seed(N)
    check(x, kv_lens=kv, key_mask=torch.rand(B, M, generator=g) < 0.7)


def test_ragged_batch():
    x = inputs(4, 4, 2, 600, 300, seed=4)
    check(x, q_lens=torch.tensor([600, 1, 0, 257], dtype=torch.int32), kv_lens=torch.tensor([1, 300, 77, 0], dtype=torch.int32))
    check(x, q_lens=torch.tensor([9999, -5, 256, 255], dtype=torch.int32), kv_lens=torch.tensor([-1, 9999, 128, 129], dtype=torch.int32))


@pytest.mark.parametrize("B,H,Hk,N,M", [(1, 6, 1, 700, 130), (2, 4, 1, 900, 1), (1, 8, 2, 333, 333), (1, 3, 1, 1500, 260),
                                        (1, 1, 1, 2600, 150), (2, 2, 1, 1300, 40), (1, 1, 1, 2300, 2300), (1, 2, 2, 300, 4000)])
def test_walks_in_pieces(B, H, Hk, N, M):
    """Few keys under many rows and few rows over many keys: dq, dk and dv are summed in pieces and joined."""
    x = inputs(B, H, Hk, N, M, seed=5)
    check(x)
    g = torch.Generator().manual_seed(M)
    check(x, q_lens=torch.tensor([N, N // 3][:B], dtype=torch.int32), kv_lens=torch.tensor([M // 2, M][:B], dtype=torch.int32),
          key_mask=torch.rand(B, M, generator=g) < 0.8)


@pytest.mark.parametrize("N", [1, 200, 600])
def test_peaked_rows(N):
    """1 % of the keys times 8: scores of 90 and more, maxima that come late."""
    check(inputs(1, 2, 1, N, 400, seed=5, boost=True))


@pytest.mark.parametrize("N", [1, 300])
def test_maxima_far_above_the_first_keys(N):
    """Keys late in the sequence whose scores are hundreds above the first tile's."""
    x = inputs(1, 2, 1, N, 2000, seed=7)
    x["k"][:, :, 1500:1503] *= 64
    x["k"][:, :, 333] *= 24
    check(x)


@pytest.mark.parametrize("N", [1, 300])
def test_large_values_under_late_maxima(N):
    """Values of 2^90 whose products with P of 2^60 would leave fp32: scores are held to the rows' own maxima."""
    x = inputs(1, 1, 1, N, 100, seed=8)
    x["v"] = (x["v"].float() * 2.0 ** 90).bfloat16()
    x["k"][:, :, 70] *= 24
    ref = reference(x)[0]
    y = {n: t.cuda() for n, t in x.items()}
    near(sol.cross_attn_fwd(y["q"], y["k"], y["v"]).double() * 2.0 ** -90, ref * 2.0 ** -90)


@pytest.mark.parametrize("scale", [1e-30, 0.01, 1.0])
def test_scales(scale):
    check(inputs(1, 2, 1, 5, 300, seed=9), scale=scale)
    check(inputs(1, 2, 1, 300, 100, seed=9), scale=scale)


@pytest.mark.parametrize("order", [(0, 2, 1, 3), (1, 0, 2, 3), (2, 0, 1, 3)])
def test_strides(order):
    back = [order.index(i) for i in range(4)]
    place = lambda t: t.permute(*order).contiguous().permute(*back)  # noqa: E731
    x = inputs(2, 4, 2, 300, 100, seed=10)
    check(x, place=place)
    wide = lambda t: torch.cat([t, torch.full_like(t, float("nan"))], -1)[..., :D]  # noqa: E731
    check(x, place=wide, kv_lens=torch.tensor([100, 33], dtype=torch.int32))
    check(inputs(2, 4, 2, 2, 900, seed=10), place=place, key_mask=torch.arange(1800).reshape(2, 900) % 3 > 0)


def test_packed_states():
    """k and v in an encoder projection [B, M, 2, Hk, D], gradients into one of the same shape."""
    B, H, Hk, N, M = 2, 4, 2, 270, 90
    x = inputs(B, H, Hk, N, M, seed=11)
    kv = torch.stack([x["k"].transpose(1, 2), x["v"].transpose(1, 2)], 2).contiguous().cuda()
    k, v = (kv[:, :, i].transpose(1, 2) for i in (0, 1))
    dkv = torch.zeros_like(kv)
    dk, dv = (dkv[:, :, i].transpose(1, 2) for i in (0, 1))
    q, do = x["q"].cuda(), x["do"].cuda()
    out, left, lse = sol.cross_attn_fwd(q, k, v, training=True)
    want = sol.cross_attn_fwd(q, x["k"].cuda(), x["v"].cuda())
    assert torch.equal(out, want)
    got = sol.cross_attn_bwd(do, q, k, v, out, left, lse, dk=dk, dv=dv)
    want = sol.cross_attn_bwd(do, q, x["k"].cuda(), x["v"].cuda(), out, left, lse)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and got[1] is dk


def test_states_shared_by_a_batch():
    """One prompt for all sequences (a stride of 0): gradients of their own, which a caller sums."""
    x = inputs(3, 2, 1, 290, 70, seed=12)
    x["k"], x["v"] = (t[:1].expand(3, -1, -1, -1).contiguous() for t in (x["k"], x["v"]))
    y = {n: t.cuda() for n, t in x.items()}
    out, left, lse = sol.cross_attn_fwd(y["q"], y["k"], y["v"], training=True)
    k, v = (y[n][:1].expand(3, -1, -1, -1) for n in ("k", "v"))
    assert k.stride(0) == 0 and torch.equal(sol.cross_attn_fwd(y["q"], k, v), out)
    a = sol.cross_attn_bwd(y["do"], y["q"], k, v, out, left, lse)
    b = sol.cross_attn_bwd(y["do"], y["q"], y["k"], y["v"], out, left, lse)
    assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_gradients_against_differences():
    """The definition that the tests above use, a step of each input both ways."""
    x = inputs(2, 4, 2, 5, 9, seed=13)
    masks = dict(kv_lens=torch.tensor([9, 4], dtype=torch.int32), key_mask=torch.arange(18).reshape(2, 9) % 4 != 1)
    grads = reference(x, **masks)[1]
    gen = torch.Generator().manual_seed(1)
    for name, grad in zip("qkv", grads):
        step = torch.randn(x[name].shape, generator=gen, dtype=torch.float64)

        def f(e):
            return (reference({**x, name: x[name].double() + e * step}, **masks)[0] * x["do"].double()).sum()
        assert abs((f(1e-5) - f(-1e-5)) / 2e-5 - (grad * step).sum()) <= 1e-7 * (grad * step).abs().sum()


def test_binding_refusals():
    x = {n: t.cuda() for n, t in inputs(2, 4, 2, 10, 20).items()}
    ok = dict(q=x["q"], k=x["k"], v=x["v"])
    sol.cross_attn_fwd(**ok)
    mask = torch.ones(2, 20, dtype=torch.bool, device="cuda")
    sol.cross_attn_fwd(key_mask=mask, **ok)
    for bad in (dict(q=x["q"].float()), dict(v=x["v"][:, :1]), dict(k=x["k"].cpu()), dict(key_mask=mask[:, :19]),
                dict(key_mask=mask.float()), dict(key_mask=mask.t()), dict(kv_lens=torch.zeros(2, device="cuda")),
                dict(q_lens=torch.zeros(2, dtype=torch.int32)), dict(out=x["q"].float()), dict(q=x["q"][..., :64])):
        with pytest.raises((TypeError, ValueError, sol.SolError)):
            sol.cross_attn_fwd(**{**ok, **bad})
    for bad in (dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(out=x["q"])):
        with pytest.raises(sol.SolError):
            sol.cross_attn_fwd(**{**ok, **bad})
    with pytest.raises(ValueError):
        sol.cross_attn_bwd(x["do"], x["q"], x["k"], x["v"], x["do"], None, None)
