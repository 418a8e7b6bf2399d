"""The differential attention's gradients on the GPU, value by value, against the
definition in 64 bits: each value has an allowance of its own.

What the kernels round (to bf16, so by at most r = 2^-8 of a term, r / sqrt(3) in
the mean square, independently of one another):
  dv: the terms (P_0 - lambda P_1) dout of a value's sum;
  dq, dk: the terms dS k, dS q;  and delta_s, one number a row, from an output of
  rounded P divided by the sum of the rounded ones, off by sum_j e_j P_j (X_j -
  delta), whose variance is r^2 / 3 sum P^2 (X - delta)^2, and from outputs kept in
  two bf16 parts, off by 2^-17 |dout| (|o_s| + |out|) a term: it enters dq[i] as
  -scale sum_j P_ij k_j and dk[j] through every row as -scale P_ij q_i (times -lambda
  for the second map);
  the result once, by r of its value.
fp32 arithmetic, coherent over a value's terms: the exponents' error, some 2^-24 of
the largest score, so 2^-21 (1 + max |score|) of the sum of the terms' sizes is
allowed.  A value may be off by six standard deviations of the sum of its independent
parts, its own rounding and that; all of them together by 1.5 times the root of the
sum of the variances (which takes every rounding as if at a binade's low end, so that
about 0.75 is expected)."""
import pytest
import torch

from paper_2609_35110_amd import sol
from test_gpu_diff_attn import inputs, maps

pytestmark = pytest.mark.gpu
D = 128
R2 = (2.0 ** -8) ** 2 / 3


def gradients(x, scale, **kw):
    """(value, variance, size of terms) of dq, dk and dv, and max |score|; on the device that x is on."""
    B, H2, N, _ = x["q"].shape
    Hv, Hk, M, H = x["v"].shape[1], x["k"].shape[1], x["v"].shape[2], H2 // 2
    p, _, q, k, valid, kl, s = maps(x, scale, **kw)
    p, q, k, valid, s = (t.cuda() for t in (p, q, k, valid, s))
    keys = (torch.arange(M) < kl[:, None]).cuda()[:, None, :, None]
    v = torch.where(keys, x["v"].cuda().double().repeat_interleave(H // Hv, 1), 0.0)
    do = torch.where(valid, x["do"].cuda().double(), 0.0)
    q = torch.where(valid[:, None], q, 0.0)
    lam = x["lam"].cuda().double()[:, None, None]
    w = torch.stack([torch.ones_like(lam), -lam])[None] * scale
    o = p @ v[:, None]
    out = o[:, 0] - lam * o[:, 1]
    X = (do @ v.transpose(-1, -2).contiguous())[:, None]
    delta = (o * do[:, None]).sum(-1, keepdim=True)
    dS = p * (X - delta) * w
    vd = R2 * ((p * (X - delta)) ** 2).sum(-1, keepdim=True)
    vd = vd + (2.0 ** -17) ** 2 * ((do.abs()[:, None] * (o.abs() + out.abs()[:, None])) ** 2).sum(-1, keepdim=True)
    vd = vd * w ** 2
    t = lambda z: z.transpose(-1, -2).contiguous()  # noqa: E731
    rows = lambda z: z.transpose(1, 2).reshape(B, H2, N, D)  # noqa: E731

    def shared(z):  # [B, 2, H, M, D] to the heads of k
        z = z.reshape(B, 2, Hv, H // Hv, M, D).sum(3).transpose(1, 2)
        return z.sum(2) if Hk == Hv else z.reshape(B, Hk, M, D)

    def values(z):
        return z.reshape(B, Hv, H // Hv, M, D).sum(2)

    P = p[:, 0] - lam * p[:, 1]
    return {"dq": (rows(dS @ k), rows(R2 * (dS ** 2 @ k ** 2) + vd * (p @ k) ** 2), rows(dS.abs() @ k.abs())),
            "dk": (shared(t(dS) @ q), shared(t(R2 * dS ** 2 + vd * p ** 2) @ q ** 2), shared(t(dS.abs()) @ q.abs())),
            "dv": (values(t(P) @ do), values(R2 * t(P ** 2) @ do ** 2), values(t(P.abs()) @ do.abs()))}, \
        s[torch.isfinite(s)].abs().max().item()


def compare(x, scale=D ** -0.5, **kw):
    want, top = gradients(x, scale, **kw)
    y = {n: t.cuda() for n, t in x.items()}
    lens = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in kw.items()}
    args = (y["q"], y["k"], y["v"], y["lam"])
    fwd = sol.diff_attn_fwd(*args, scale=scale, training=True, **lens)
    got = sol.diff_attn_bwd(y["do"], *args, *fwd, scale=scale, **lens)
    for (name, (ref, var, size)), a in zip(want.items(), got):
        d = (a.double() - ref).abs()
        assert torch.isfinite(d).all()
        exact = 2.0 ** -21 * (1 + top) * size
        over = d - (6 * var.sqrt() + 2.0 ** -8 * ref.abs() + exact)
        part = (d.norm() / (var + R2 * ref ** 2).sum().sqrt().clamp(min=1e-30)).item()
        print(name, "norm over the variances' root %.3f, allowance of the rms %.4f" % (
            part, ((6 * var.sqrt() + exact).norm() / ref.norm().clamp(min=1e-30)).item()), flush=True)
        assert (over <= 0).all(), (name, over.max())
        assert d.norm() <= 1.5 * (var + R2 * ref ** 2).sum().sqrt() + exact.norm(), name


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,H,Hv,own_keys,N,M", [
    (1, 2, 1, True, 1, 40), (2, 3, 3, True, 65, 127), (1, 2, 1, False, 257, 300), (2, 6, 1, False, 700, 130),
    (1, 8, 2, True, 333, 333), (1, 1, 1, True, 2300, 2300), (1, 2, 2, False, 1900, 1900), (1, 1, 1, True, 2600, 150)])
def test_each_value(B, H, Hv, own_keys, N, M, causal):
    compare(inputs(B, H, Hv, own_keys, N, M, seed=N + M), causal=causal)


@pytest.mark.parametrize("own_keys", [False, True])
def test_each_value_of_peaked_rows(own_keys):
    compare(inputs(1, 2, 1, own_keys, 200, 400, seed=5, boost=True))


def test_each_value_of_a_ragged_batch():
    x = inputs(3, 4, 2, True, 500, 600, seed=2)
    compare(x, causal=True, q_lens=torch.tensor([500, 1, 77], dtype=torch.int32),
            kv_lens=torch.tensor([333, 600, 64], dtype=torch.int32))


def test_a_wrong_row_is_found():
    """The allowances themselves: a key's row left at zero, or one value off by a tenth of its row's rms, passes none of them."""
    x = inputs(2, 6, 1, False, 700, 130, seed=830)
    want, top = gradients(x, D ** -0.5)
    for name, (ref, var, size) in want.items():
        allowed = 6 * var.sqrt() + 2.0 ** -8 * ref.abs() + 2.0 ** -21 * (1 + top) * size
        rms = ref.norm(dim=-1, keepdim=True) / D ** 0.5
        assert (allowed < 0.1 * torch.maximum(rms, ref.abs())).float().mean() > 0.99, name
        assert (allowed.norm(dim=-1) < ref.norm(dim=-1)).all(), name
