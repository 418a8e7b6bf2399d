"""Queries and keys normalised and rotated at positions of their own, on the GPU,
against the definition in 64 bits (plain torch on the CPU), through the torch binding.

Tolerances.  An output is fp32 arithmetic rounded once to bf16: the sum of 128 squares
in a chain of 8 and a tree of 4 (12 roundings, half of them count under the root), the
square root, the reciprocal, two products: fewer than 16 roundings of 2^-24 each before
the rotation (whose own are 2^-47), so a value may be off by half a bf16 step, 2^-8 of
its size at most, and 2^-20 of its pair's: within a pair of components up to the pair's
length.  A gradient: n = R^T dy is two products and one sum with cosines rounded to
2^-24; h, xh, the mean of 128 products h xh and dx three products: fewer than 40
roundings, each of terms no larger than r (|h| + |xh| mean |h xh|): 2^-18 of that, and
half a step.  A weight's gradient is an fp32 sum of terms n xh, a chain of them in a
thread, then 16, then 64 bits: held to 2^-24 x (terms of a chain + 16 + 8 of each term)
of the sum of the terms' sizes.  A term's size is its pair's, |xh| sqrt(a^2 + b^2): n is
a c + b s, two products of which each may be as large as the pair and whose roundings
stay when they cancel (n = 0 has an error of 2^-24 of the pair's size, not of its own)."""
import math

import pytest
import torch

from paper_2609_35110_amd import sol

pytestmark = pytest.mark.gpu
D = 128
BF16 = 2.0 ** -8
STREAM_WGS = 2048


def inputs(B, H, Hk, N, seed=0, T=9, Hl=5, Wl=7, text=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda h: torch.randn(B, h, N, D, generator=g).bfloat16()  # noqa: E731
    pos = torch.stack([torch.randint(0, n, (B, N), generator=g) for n in (T, Hl, Wl)], -1).int()
    pos[:, :text] = -1
    return {"q": r(H), "k": r(Hk) if Hk else None, "gq": 1 + 0.3 * torch.randn(D, generator=g),
            "gk": 1 + 0.3 * torch.randn(D, generator=g) if Hk else None, "dq": r(H), "dk": r(Hk) if Hk else None,
            "pos": pos, "grid": (T, Hl, Wl)}


def turns(pos, split):
    """The angle of each pair, [B, 1, N, D / 2] in 64 bits; none where the coordinate is below 0 or past the split."""
    B, N, _ = pos.shape
    a = torch.zeros(B, N, D // 2, dtype=torch.float64)
    at = 0
    for axis, d in enumerate(split):
        steps = 10000.0 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d) if d else torch.zeros(0)
        a[..., at:at + d // 2] = pos[..., axis, None].clamp(min=0).double() * steps
        at += d // 2
    return a[:, None]


def turn(x, a):
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack([x0 * a.cos() - x1 * a.sin(), x0 * a.sin() + x1 * a.cos()], -1).flatten(-2)


def definition(x, dy, gamma, a, eps):
    """y, dx, dgamma's terms, and the sizes that the allowances go by."""
    x, dy = x.double(), dy.double()
    n = turn(dy, -a)
    pair = lambda z: (z.reshape(*z.shape[:-1], D // 2, 2).norm(dim=-1, keepdim=True).expand(*z.shape[:-1], D // 2, 2)).flatten(-2)  # noqa: E731
    if gamma is None:
        y = turn(x, a)
        return y, n, None, pair(x), pair(dy), None
    r = ((x * x).mean(-1, keepdim=True) + eps) ** -0.5
    xh, h = x * r, n * gamma.double()
    y = turn(xh * gamma.double(), a)
    dx = r * (h - xh * (h * xh).mean(-1, keepdim=True))
    size = pair(dy) * gamma.double().abs()
    return y, dx, n * xh, pair(xh * gamma.double()), r * (size + xh.abs() * (size * xh.abs()).mean(-1, keepdim=True)), pair(dy) * xh.abs()


def check(x, eps=1e-6, split=(32, 48, 48), lens=None, norm=(True, True), place=lambda t: t, base=None, positions=True):
    """Both directions against the definition; place: how a tensor lies in device memory (a view of its values)."""
    B, H, N, _ = x["q"].shape
    T, Hl, Wl = x["grid"]
    inside = torch.ones(B, N, dtype=torch.bool) if lens is None else torch.arange(N) < lens.clamp(0, N)[:, None]
    inside = inside[:, None, :, None]
    pos = (base or (lambda p: p))(x["pos"]).cuda() if positions else None
    tab = sol.rope3d_table(T, Hl, Wl, split=split)
    a = turns(x["pos"] if positions else torch.full_like(x["pos"], -1), split)
    y = {n: place(t.cuda()) if t is not None and t.dim() == 4 else t for n, t in x.items() if isinstance(t, torch.Tensor) or t is None}
    gq, gk = (g.cuda() if on and g is not None else None for g, on in zip((x["gq"], x["gk"]), norm))
    dl = None if lens is None else lens.cuda()
    where = (pos, T, Hl, Wl, tab)
    opts = dict(q_gamma=gq, k_gamma=gk, eps=eps, lens=dl, split=split)
    fill = lambda t: None if t is None else torch.full_like(t, 7.0)  # noqa: E731
    outs = sol.qk_norm_rope(y["q"], y["k"], *where, q_out=fill(y["q"]), k_out=fill(y["k"]), **opts)
    grads = sol.qk_norm_rope_bwd(y["dq"], y["dk"], y["q"], y["k"], *where, **opts)
    again = sol.qk_norm_rope_bwd(y["dq"], y["dk"], y["q"], y["k"], *where, **opts)
    for g1, g2 in zip(grads, again):
        assert (g1 is None and g2 is None) or torch.equal(g1, g2)
    for i, (t, dy, gamma) in enumerate(((x["q"], x["dq"], gq), (x["k"], x["dk"], gk))):
        if t is None:
            assert outs[i] is None and grads[i] is None and grads[2 + i] is None
            continue
        ref, dx, terms, size, dsize, tsize = definition(t, dy, None if gamma is None else gamma.cpu(), a, eps)
        got, dgot = outs[i].cpu().double(), grads[i].cpu().double()
        keep = inside.expand_as(got)
        assert (got[~keep] == 7.0).all() and (dgot[~keep] == 0).all()
        over = (got - ref).abs() - (BF16 * ref.abs() + 2.0 ** -20 * size)
        assert (over[keep] <= 0).all(), over[keep].max()
        over = (dgot - dx).abs() - (BF16 * dx.abs() + 2.0 ** -18 * dsize)
        assert (over[keep] <= 0).all(), over[keep].max()
        if gamma is None:
            assert grads[2 + i] is None
            continue
        terms = torch.where(inside, terms, 0.0)
        chain = t.shape[1] * -(-B * N // (16 * min(STREAM_WGS, -(-B * N // 16))))  # (all heads of a tile in one thread: the most)
        off = (grads[2 + i].cpu().double() - terms.sum((0, 1, 2))).abs()
        assert (off <= 2.0 ** -24 * (chain + 24) * torch.where(inside, tsize, 0.0).sum((0, 1, 2))).all()
    return outs, grads


SHAPES = [(1, 1, 0, 1), (1, 1, 1, 1), (32, 24, 8, 1), (1, 3, 1, 17), (2, 2, 5, 33), (3, 4, 2, 100), (1, 40, 40, 65), (5, 7, 0, 13)]


@pytest.mark.parametrize("norm", [(True, True), (False, False), (True, False)])
@pytest.mark.parametrize("B,H,Hk,N", SHAPES)
def test_against_definition(B, H, Hk, N, norm):
    check(inputs(B, H, Hk, N, seed=N, text=min(3, N // 2)), norm=norm)


@pytest.mark.parametrize("split", [(128, 0, 0), (0, 64, 64), (16, 24, 24), (8, 0, 0), (0, 0, 0)])
def test_splits(split):
    check(inputs(2, 3, 2, 40, seed=4), split=split)


def test_ragged_batch():
    x = inputs(4, 3, 2, 50, seed=5)
    check(x, lens=torch.tensor([50, 1, 0, 33], dtype=torch.int32))
    check(x, lens=torch.tensor([999, -3, 16, 49], dtype=torch.int32), norm=(False, False))


def test_no_positions():
    check(inputs(2, 3, 2, 40, seed=6), positions=False)
    check(inputs(2, 3, 2, 40, seed=6), positions=False, norm=(False, True))


@pytest.mark.parametrize("order", [(0, 2, 1, 3), (1, 0, 2, 3), (2, 0, 1, 3)])
def test_strides(order):
    """Rows that lie token by token, head by head, batch innermost; and a row apart."""
    back = [order.index(i) for i in range(4)]
    x = inputs(3, 4, 2, 21, seed=7)
    check(x, place=lambda t: t.permute(*order).contiguous().permute(*back))
    wide = lambda t: torch.cat([t, torch.full_like(t, float("nan"))], -1)[..., :D]  # noqa: E731
    check(x, place=wide, lens=torch.tensor([21, 4, 20], dtype=torch.int32))


def test_packed_projection_in_place():
    """q and k inside [B, N, 3, H, D]: read there, and written back there; v is left alone."""
    x = inputs(2, 5, 5, 30, seed=8)
    qkv = torch.randn(2, 30, 3, 5, D).bfloat16().cuda()
    views = [qkv[:, :, i].transpose(1, 2) for i in range(3)]
    views[0].copy_(x["q"])
    views[1].copy_(x["k"])
    v = views[2].clone()
    T, Hl, Wl = x["grid"]
    where = (x["pos"].cuda(), T, Hl, Wl, sol.rope3d_table(T, Hl, Wl))
    opts = dict(q_gamma=x["gq"].cuda(), k_gamma=x["gk"].cuda())
    want = sol.qk_norm_rope(x["q"].cuda(), x["k"].cuda(), *where, **opts)
    got = sol.qk_norm_rope(views[0], views[1], *where, q_out=views[0], k_out=views[1], **opts)
    assert got[0] is views[0] and torch.equal(views[0], want[0]) and torch.equal(views[1], want[1])
    assert torch.equal(views[2], v)
    # the gradients in place too
    x0, x1 = x["q"].cuda(), x["k"].cuda()
    want = sol.qk_norm_rope_bwd(x["dq"].cuda(), x["dk"].cuda(), x0, x1, *where, **opts)
    views[0].copy_(x["dq"])
    views[1].copy_(x["dk"])
    got = sol.qk_norm_rope_bwd(views[0], views[1], x0, x1, *where, dq=views[0], dk=views[1], **opts)
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and torch.equal(views[2], v)


@pytest.mark.parametrize("norm", [False, True])
def test_raster_positions_are_the_raster_rotation(norm):
    """The positions of a grid with text ahead give sol_qknorm_rope3d's bits."""
    T, Hl, Wl, text = 3, 6, 7, 5
    N = text + T * Hl * Wl
    x = inputs(2, 3, 3, N, seed=9)
    n = torch.arange(N) - text
    pos = torch.where(n[:, None] < 0, -1, torch.stack([n // (Hl * Wl), n // Wl % Hl, n % Wl], -1)).int().cuda()
    for split in ((32, 48, 48), (16, 24, 24)):
        tab = sol.rope3d_table(T, Hl, Wl, split=split)
        gamma = x["gq"].cuda() if norm else None
        q = x["q"].cuda()
        want = sol.qknorm_rope3d(q, T, Hl, Wl, tab, gamma, split=split)
        got, _ = sol.qk_norm_rope(q, None, pos, T, Hl, Wl, tab, q_gamma=gamma, split=split)
        assert torch.equal(got, want)
        # a table whose extents only bound the coordinates
        big = sol.rope3d_table(T + 9, Hl + 1, Wl + 4, split=split)
        got, _ = sol.qk_norm_rope(q, None, pos.expand(2, N, 3).contiguous(), T + 9, Hl + 1, Wl + 4, big, q_gamma=gamma, split=split)
        assert torch.equal(got, want)


def test_far_positions():
    x = inputs(1, 2, 1, 64, seed=10, T=1_000_003, Hl=70_001, Wl=5)
    check(x)


def test_coordinates_past_the_table():
    """A token's rows are NaN and no others; an axis without dims is not asked; a weight's gradient is NaN."""
    x = inputs(2, 3, 2, 40, seed=11)
    T, Hl, Wl = x["grid"]
    good = x["pos"].cuda()
    tab = sol.rope3d_table(T, Hl, Wl)
    opts = dict(q_gamma=x["gq"].cuda(), k_gamma=x["gk"].cuda())
    q, k = x["q"].cuda(), x["k"].cuda()
    want = sol.qk_norm_rope(q, k, good, T, Hl, Wl, tab, **opts)
    wantg = sol.qk_norm_rope_bwd(x["dq"].cuda(), x["dk"].cuda(), q, k, good, T, Hl, Wl, tab, **opts)
    for axis, value in ((0, T), (1, 2 ** 31 - 1), (2, Wl + 3)):
        pos = good.clone()
        pos[1, 17, axis] = value
        got = sol.qk_norm_rope(q, k, pos, T, Hl, Wl, tab, **opts)
        grads = sol.qk_norm_rope_bwd(x["dq"].cuda(), x["dk"].cuda(), q, k, pos, T, Hl, Wl, tab, **opts)
        for a, b in zip(got + grads[:2], want + wantg[:2]):
            bad = torch.isnan(a)
            assert bad[1, :, 17].all() and bad.sum() == a.shape[1] * D
            assert torch.equal(a[~bad], b[~bad])
        assert torch.isnan(grads[2]).all() and torch.isnan(grads[3]).all()
        outside = sol.qk_norm_rope_bwd(x["dq"].cuda(), x["dk"].cuda(), q, k, pos, T, Hl, Wl, tab,
                                       lens=torch.tensor([40, 17], dtype=torch.int32).cuda(), **opts)
        assert all(torch.isfinite(t).all() for t in outside)  # (a token behind its sequence is not looked at)
    pos = good.clone()
    pos[..., 2] = 2 ** 31 - 1
    tab = sol.rope3d_table(T, Hl, 0, split=(64, 64, 0))
    got = sol.qk_norm_rope(q, k, pos, T, Hl, 0, tab, split=(64, 64, 0), **opts)
    assert all(torch.isfinite(t).all() for t in got)


def test_negative_axes_alone():
    """An image has rows and columns but no frame: one coordinate below 0."""
    x = inputs(2, 2, 2, 33, seed=12)
    x["pos"][..., 0] = -1
    x["pos"][1, :, 2] = -2 ** 31
    check(x)


def test_zero_rows_and_eps():
    x = inputs(1, 2, 1, 20, seed=13)
    x["q"][:, :, 3] = 0
    check(x)
    check(x, eps=0.25)
    T, Hl, Wl = x["grid"]
    tab = sol.rope3d_table(T, Hl, Wl)
    out, _ = sol.qk_norm_rope(x["q"].cuda(), None, x["pos"].cuda(), T, Hl, Wl, tab, q_gamma=x["gq"].cuda(), eps=0.0)
    assert torch.isnan(out[:, :, 3]).all() and torch.isfinite(out[:, :, 4:]).all()


def test_long_walks_of_a_workgroup():
    """More tiles than workgroups: each walks several, and sums its weights' gradients over them."""
    check(inputs(1, 1, 1, 16 * STREAM_WGS + 16 * 700 + 5, seed=14))


def test_gradients_against_differences():
    """A step of each input's direction, both ways, in the definition that the tests above use."""
    x = inputs(1, 2, 1, 6, seed=15)
    a = turns(x["pos"], (32, 48, 48))
    gen = torch.Generator().manual_seed(1)
    for t, dy, gamma in ((x["q"], x["dq"], x["gq"]), (x["k"], x["dk"], x["gk"])):
        y, dx, terms, _, _, _ = definition(t, dy, gamma, a, 1e-6)
        step = torch.randn(t.shape, generator=gen, dtype=torch.float64)
        f = lambda e: (definition(t.double() + e * step, dy, gamma, a, 1e-6)[0] * dy.double()).sum()  # noqa: E731
        assert abs((f(1e-5) - f(-1e-5)) / 2e-5 - (dx * step).sum()) <= 1e-7 * (dx * step).abs().sum()
        step = torch.randn(D, generator=gen, dtype=torch.float64)
        f = lambda e: (definition(t, dy, gamma.double() + e * step, a, 1e-6)[0] * dy.double()).sum()  # noqa: E731
        assert abs((f(1e-5) - f(-1e-5)) / 2e-5 - (terms.sum((0, 1, 2)) * step).sum()) <= 1e-7 * (terms * step).abs().sum()


def test_binding_refusals():
    x = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in inputs(2, 3, 2, 10).items()}
    T, Hl, Wl = x["grid"]
    tab = sol.rope3d_table(T, Hl, Wl)
    ok = dict(q=x["q"], k=x["k"], pos=x["pos"], T=T, Hl=Hl, Wl=Wl, table=tab)
    sol.qk_norm_rope(**ok)
    for bad in (dict(q=x["q"].float()), dict(k=x["k"][:, :, :9]), dict(pos=x["pos"].long()), dict(pos=x["pos"][:, :9]),
                dict(pos=x["pos"].cpu()), dict(table=tab[:-4]), dict(T=T + 1), dict(table=sol.rope3d_table(T, Hl, Wl + 1)),
                dict(q_gamma=x["gq"].bfloat16()), dict(lens=torch.zeros(3, dtype=torch.int32, device="cuda")),
                dict(k=None, k_out=x["k"]), dict(q=x["q"][..., :64])):
        with pytest.raises((TypeError, ValueError, sol.SolError)):
            sol.qk_norm_rope(**{**ok, **bad})
    for bad in (dict(table=None), dict(eps=-1.0), dict(eps=math.nan), dict(q_out=x["k"].new_empty(2, 3, 10, D)[:, :1].expand(2, 3, 10, D))):
        with pytest.raises(sol.SolError):
            sol.qk_norm_rope(**{**ok, **bad})
