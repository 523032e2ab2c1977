"""Values at the ends of their types' range in the 8-bit cache and its attention."""

import pytest
import torch

import paper_2509_05165_b200 as kvc
from test_gpu_decode import E4, I8, _bits, _gen, dev  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [I8, E4])
def test_evict_blocks_of_the_largest_exponent(dev, fmt):
    """Codes that stand for more than fp32 holds (448 * 2^121): moved with their exponent, as its definition says."""
    g = _gen(7)
    c = kvc.alloc_cache(1, 2, 64, 64, 32, fmt, dev)
    top = 448.0 if fmt == E4 else 127.0
    x = (torch.randn((1, 2, 64, 64), generator=g) * top / 4).clamp(-top, top)
    x[..., 0] = top
    for t in (c.k, c.v):
        t.copy_(x.round().to(I8) if fmt == I8 else x.to(E4))
    for t in (c.k_exp, c.v_exp):
        t.fill_(121)
    c.lengths.fill_(64)
    dst, idx = kvc.alloc_cache(1, 2, 64, 40, 16, fmt, dev), torch.empty((1, 2, 40), dtype=torch.int32, device=dev)
    kvc.kvc_evict(c, dst, torch.rand((1, 2, 64), generator=g).to(dev), 40, 5, idx)
    for j in range(2):
        kept = idx[0, j].long()
        for a, b in ((c.k, dst.k), (c.v, dst.v)):
            assert torch.equal(_bits(b)[0, j], _bits(a)[0, j][kept])
    assert (dst.k_exp[..., :3] == 121).all() and (dst.v_exp[..., :3] == 121).all()
