"""Attention over caches so long that a warp goes on for dozens of steps (exponents are read 32 steps at a time), with one, two
and four tiles of query rows, against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2509_05165_b200 as kvc
from test_gpu_decode import BF, E4, F32, I8, _check_attend, _filled_cache, _gen, dev  # noqa: F401

pytestmark = pytest.mark.gpu

LONG = [
    # batch, KV heads, query heads per KV head, rows, d, tokens, block, format, type
    (8, 8, 2, 1, 64, 32768, 16, I8, BF),            # shares that lie within a head, and CTAs that hold the ends of two: 55 steps
    (8, 8, 1, 1, 64, 32768, 128, E4, F32),
    (1, 2, 7, 4, 64, 700001, 32, E4, BF),           # 28 rows: four tiles; 37 steps
    (1, 2, 4, 4, 64, 650001, 64, I8, BF),           # 16 rows: two tiles
    (1, 2, 4, 4, 64, 650001, 16, E4, F32),
    (1, 2, 7, 4, 128, 131073, 64, I8, BF),
    (1, 1, 16, 1, 128, 131071, 16, E4, F32),
]


@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("b,h,G,rows,d,n,block,fmt,dtype", LONG)
def test_attend_for_many_steps_per_warp(dev, b, h, G, rows, d, n, block, fmt, dtype, weights):
    """Tolerances as derived in _check_attend: the sums of a warp, its CTA and the parts are under a hundred fp32 additions one after
    another for a term, 2^-17 relatively, which the share of the logits' errors (2^-18 of sum |q k| scale, above 4 here) covers."""
    g = _gen(n + rows)
    lengths = torch.full((b, h), n)
    lengths[0, 0] -= 77
    c = _filled_cache(dev, g, b, h, d, n + 5, block, fmt, lengths)
    q = torch.randn((b, h * G, rows, d), generator=g).to(dtype).to(dev)
    out, lse = torch.full_like(q, math.nan), torch.full((b, h * G, rows), math.nan, device=dev)
    w0 = torch.rand((b, h, n + 5), generator=g).to(dev) if weights else None
    weight = torch.full((b, h, n + 5), -9.0, device=dev) if weights else None
    ws = torch.full((kvc.kvc_attend_workspace_size(c, q, weights),), 0xFF, dtype=torch.uint8, device=dev)
    kvc.kvc_attend(c, q, out, lse, weight=w0, weight_out=weight, workspace=ws)
    for i in sorted({0, b // 2, b - 1}):
        s = slice(i, i + 1)
        one = kvc.Cache(c.k[s], c.v[s], c.k_exp[s], c.v_exp[s], c.lengths[s], block)
        _check_attend(one, q[s], out[s], lse[s], weight[s] if weights else None, w0[s] if weights else None, True, d ** -0.5)
    if weights:
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
