"""Cross attention in tiles of 256 rows whose last one ends inside a wave's 64, on the
GPU: the waves behind hold the last row again and store none of it, since the wave that
has it may walk its rows a second time, under other maxima, for any one of them.
Tolerances: test_gpu_cross_attn.py's."""
import math

import pytest
import torch

from paper_2609_35110_amd import sol
from test_gpu_cross_attn import D, check, inputs
from test_gpu_cross_tiles import some_mask

pytestmark = pytest.mark.gpu


def late(B, H, Hk, N, M, lens, seed):
    """Ordinary inputs, but that one row other than the last one of the wave that has the last has a score hundreds
    above its first keys' near the last key: 3 |k|^2 / sqrt(D) = 543 for a k of size 4."""
    x = inputs(B, H, Hk, N, M, seed=seed)
    x["k"][:, :, M - 20] *= 4
    for b, n in enumerate(lens):
        first = (n - 1) // 64 * 64  # of the wave that has the last row
        row = first if n - 1 - first < 32 or b % 2 else n - 2
        if row < n - 1:
            x["q"][b, :, row] = (3 * x["k"][b, :, M - 20].float()).bfloat16().repeat_interleave(H // Hk, 0)
    return x


# whole tiles
WHOLE = [(2, 24, 24, 266, 300, None), (1, 30, 6, 330, 513, None), (3, 24, 8, 300, 290, [258, 299, 266]),
         (4, 24, 24, 200, 300, [2, 64, 65, 130]), (3, 22, 22, 600, 290, [580, 514, 640])]


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("B,H,Hk,N,M,lens", WHOLE)
def test_the_last_row_is_its_own_waves(B, H, Hk, N, M, lens, masked):
    """Against 64 bits; and every row, its rounding's rest and log sum bit for bit those of a call whose tiles are
    full, the last row in every place behind it, where no wave stores another's."""
    ends = [min(n, N) for n in lens or [N] * B]
    x = late(B, H, Hk, N, M, ends, seed=N)
    masks = {} if lens is None else dict(q_lens=torch.tensor(lens, dtype=torch.int32))
    if masked:
        masks["key_mask"] = some_mask(B, M, 0.7, M) | (torch.arange(M) >= M - 30).to(torch.uint8)
    out, _ = check(x, **masks)
    dm = {n: t.cuda() for n, t in masks.items()}
    full = torch.zeros(B, H, (N + 255) // 256 * 256, D, dtype=torch.bfloat16)
    for b, n in enumerate(ends):
        full[b, :, :n] = x["q"][b, :, :n]
        full[b, :, n:] = x["q"][b, :, n - 1:n]
    y = {n: t.cuda() for n, t in x.items()}
    dm_full = {n: t for n, t in dm.items() if n != "q_lens"}
    want = sol.cross_attn_fwd(full.cuda(), y["k"], y["v"], training=True, **dm_full)
    assert math.isfinite(want[0].float().abs().max())
    for _ in range(3):
        got = sol.cross_attn_fwd(y["q"], y["k"], y["v"], training=True, **dm)
        assert torch.equal(sol.cross_attn_fwd(y["q"], y["k"], y["v"], out=out.clone(), **dm), out)
        for a, w in zip(got, want):
            for b, n in enumerate(ends):
                assert torch.equal(a[b, :, :n], w[b, :, :n]), (b, n)


@pytest.mark.parametrize("masked", [False, True])
def test_shared_tiles_of_one_wave(masked):
    """130 heads of 40 rows over 2,100 keys: tiles that workgroups share, of one wave with rows."""
    B, H, N, M = 1, 130, 40, 2100
    x = late(B, H, H, N, M, [N], seed=1)
    check(x, **(dict(key_mask=some_mask(B, M, 0.7, M) | (torch.arange(M) >= M - 30).to(torch.uint8)) if masked else {}))
