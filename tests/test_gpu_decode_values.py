"""Values at the ends of their types' range, and rows that are not finite, in the 8-bit cache and its attention."""
import math

import pytest
import torch

import decode_ref as R
import paper_2509_05165_b200 as kvc
from test_gpu_decode import BF, E4, F32, I8, _bits, _check_attend, _filled_cache, _gen, dev  # noqa: F401

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


@pytest.mark.parametrize("fmt", [I8, E4])
def test_evict_values_next_to_the_types_largest(dev, fmt):
    """bf16's largest value rounds to 2^128 in e4m3, which fp32 does not hold: its block still takes the smallest exponent that does."""
    g = _gen(8)
    x = [R.spread_rows(g, 1, 2, 64, 64).to(BF) for _ in range(2)]
    x[0][..., 5, 3], x[1][..., 40, 60] = torch.finfo(BF).max, -torch.finfo(BF).max
    c = kvc.alloc_cache(1, 2, 64, 64, 32, fmt, dev)
    kvc.kvc_cache_append(c, x[0].to(dev), x[1].to(dev))
    w = torch.rand((1, 2, 64), generator=g)
    w[..., 5], w[..., 40] = 2.0, 2.0
    dst, idx = kvc.alloc_cache(1, 2, 64, 40, 16, fmt, dev), torch.empty((1, 2, 40), dtype=torch.int32, device=dev)
    kvc.kvc_evict(c, dst, w.to(dev), 40, 5, idx)
    held = R.cache_values(c)
    for j in range(2):
        kept = idx[0, j].cpu().long()
        for codes, exps, v in ((dst.k, dst.k_exp, held[0]), (dst.v, dst.v_exp, held[1])):
            want = R.Held(fmt, 16).fill(v[0, j][kept])
            assert exps[0, j].tolist() == want.exps
            assert torch.equal(codes[0, j].cpu().double(), torch.cat(want.codes))


# ---- rows that are not finite ------------------------------------------------------------------------------------------

def _held(x, fmt):
    """Codes and exponent of a block's rows: the exponent by the finite values; infinities take the largest code, NaN zero."""
    x = x.double()
    fin = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    e = R.exponent(float(fin.abs().max()) if x.numel() else 0.0, fmt)
    return R.round_code(torch.nan_to_num(x, nan=0.0, posinf=math.inf, neginf=-math.inf) * 2.0 ** -e, fmt), e


def _spoil(x, dtype):
    """Infinities of both signs and NaN in some rows; blocks with nothing else; the type's largest value beside others."""
    x = x.clone()
    x[..., 3, 5], x[..., 4, 0], x[..., 5, -1] = math.inf, -math.inf, math.nan
    x[..., 40, 7] = math.nan
    x[..., 128:160, :] = math.nan
    x[..., 130, :], x[..., 131, :] = math.inf, -math.inf
    x[..., 190, 1] = torch.finfo(dtype).max / 4
    x[..., 191, 2] = -math.inf
    return x


@pytest.mark.parametrize("fmt", [I8, E4])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,block", [(64, 16), (128, 32), (64, 64), (128, 128)])
def test_gather_of_rows_that_are_not_finite(dev, fmt, dtype, d, block):
    """Every value beside them keeps its place and size, and the call says so in its status; rows that are not kept do not matter."""
    h, n = 2, 300
    g = _gen(block)
    k, v = [_spoil(R.spread_rows(g, 1, h, n, d), dtype).to(dtype) for _ in range(2)]
    desc = kvc.kvc_desc_init(1, 1, h, h, d, n, 1, kvc.F32 if dtype == F32 else kvc.BF16)
    c = kvc.alloc_cache(1, h, d, n, block, fmt, dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    kvc.kvc_cache_gather(desc, [k.to(dev)], [v.to(dev)], None, None, [c], device_status=status)
    for j in range(h):
        for codes, exps, x in ((c.k, c.k_exp, k), (c.v, c.v_exp, v)):
            for r in range(-(-n // block)):
                want, e = _held(x[0, j, r * block:(r + 1) * block], fmt)
                assert int(exps[0, j, r]) == e, (j, r)
                assert torch.equal(codes[0, j, r * block:(r + 1) * block].cpu().double(), want), (j, r)
    assert int(status) == -7
    # what was there before stays but for "no error", and rows that did not fit say more
    status.fill_(-6)
    kvc.kvc_cache_gather(desc, [k.to(dev)], [v.to(dev)], None, None, [c], device_status=status)
    assert int(status) == -6
    status.zero_()
    small = kvc.alloc_cache(1, h, d, 200, block, fmt, dev)
    kvc.kvc_cache_gather(desc, [k.to(dev)], [v.to(dev)], None, None, [small], device_status=status)
    assert int(status) == -6
    status.zero_()
    idx = torch.cat([torch.arange(6, 40), torch.arange(41, 128), torch.arange(192, n), torch.arange(6), torch.tensor([40]), torch.arange(128, 192)])
    idx = idx.to(torch.int32).expand(1, 1, h, n).contiguous().to(dev)
    kvc.kvc_cache_gather(desc, [k.to(dev)], [v.to(dev)], idx, torch.full((1, 1), 229, dtype=torch.int32, device=dev), [c], device_status=status)
    assert int(status) == 0


@pytest.mark.parametrize("fmt", [I8, E4])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,block,rows", [(64, 16, 1), (128, 32, 7), (64, 128, 1), (128, 128, 130), (128, 64, 400), (64, 16, 400)])
def test_append_of_rows_that_are_not_finite(dev, fmt, dtype, d, block, rows):
    """The rows that an open block holds already are left alone, the ordinary new values beside theirs are kept."""
    b, h, have = 2, 2, block // 2 + 1
    g = _gen(rows)
    c = kvc.alloc_cache(b, h, d, have + rows + 3, block, fmt, dev)
    old = [R.spread_rows(g, b, h, have, d).to(dtype) for _ in range(2)]
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    kvc.kvc_cache_append(c, old[0].to(dev), old[1].to(dev), device_status=status)
    assert int(status) == 0
    new = [0.25 * torch.randn((b, h, rows, d), generator=g).to(dtype) for _ in range(2)]
    new[0][0, 0, 0, 3], new[0][0, 1, rows - 1, d - 1], new[1][0, 0, rows // 2, 0], new[1][0, 1, 0, 8] = math.inf, math.nan, -math.inf, math.nan
    kvc.kvc_cache_append(c, new[0].to(dev), new[1].to(dev), device_status=status, n_new=torch.tensor([rows, 0], dtype=torch.int32, device=dev))
    assert int(status) == -7
    for j in range(h):
        for codes, exps, was, x in ((c.k, c.k_exp, old[0], new[0]), (c.v, c.v_exp, old[1], new[1])):
            first, e0 = _held(was[0, j, :block], fmt)
            assert have < block
            room = min(block - have, rows)
            _, e1 = _held(x[0, j, :room], fmt)
            e = max(e0, e1)
            if e > e0:
                first = R.round_code(first * 2.0 ** max(e0 - e, -126), fmt)
            ordinary = torch.nan_to_num(x[0, j].double(), nan=0.0, posinf=math.inf, neginf=-math.inf)
            want = [torch.cat([first, R.round_code(ordinary[:room] * 2.0 ** -e, fmt)])]
            assert int(exps[0, j, 0]) == e
            for r in range(room, rows, block):
                w, e = _held(x[0, j, r:r + block], fmt)
                want.append(w)
                assert int(exps[0, j, (have + r) // block]) == e
            assert torch.equal(codes[0, j, :have + rows].cpu().double(), torch.cat(want)), j
    assert (c.lengths.cpu() == torch.tensor([[have + rows] * h, [have] * h])).all()
    # the second sequence's rows of this call are padding: NaN there is not looked at
    status.zero_()
    for x in new:
        x[0], x[1] = 0.5, math.nan
    c.lengths.fill_(1)
    kvc.kvc_cache_append(c, new[0].to(dev), new[1].to(dev), device_status=status, n_new=torch.tensor([rows, 0], dtype=torch.int32, device=dev))
    assert int(status) == 0


@pytest.mark.parametrize("fmt", [I8, E4])
def test_attention_over_rows_that_were_not_finite(dev, fmt):
    """A NaN in the last token leaves rows that do not see that token as they are, and no output is NaN: it is held as zero."""
    g = _gen(9)
    k, v = [torch.randn((1, 2, 50, 64), generator=g).to(BF) for _ in range(2)]
    k[..., 49, 3], v[..., 49, 5], k[..., 48, 0] = math.nan, math.nan, math.inf
    c = kvc.alloc_cache(1, 2, 64, 60, 16, fmt, dev)
    kvc.kvc_cache_append(c, k.to(dev), v.to(dev))
    q = torch.randn((1, 4, 3, 64), generator=g).to(BF).to(dev)
    out, lse = torch.empty_like(q), torch.empty((1, 4, 3), device=dev)
    w = torch.full((1, 2, 60), -9.0, device=dev)
    ws = torch.empty(kvc.kvc_attend_workspace_size(c, q, True), dtype=torch.uint8, device=dev)
    kvc.kvc_attend(c, q, out, lse, weight_out=w, workspace=ws)
    _check_attend(c, q, out, lse, w, torch.zeros_like(w), True, 1 / 8.0)


# ---- attention ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 3, 9])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_query_row_that_is_not_finite_gives_nan_and_no_other_row_does(dev, dtype, rows, bad):
    """Its outputs, its log-sum-exp (-inf would say that it sees no token) and the weights of its KV head; the rest is untouched."""
    g = _gen(rows)
    c = _filled_cache(dev, g, 2, 2, 64, 300, 32, I8, torch.tensor([[300, 200], [130, 0]]))
    q = torch.randn((2, 6, rows, 64), generator=g).to(dtype).to(dev)
    spoilt = q.clone()
    spoilt[0, 1, rows - 1, 7] = bad
    spoilt[1, 5, rows - 1] = bad                             # sees no token: zeros and -inf, whatever it holds
    ws = torch.empty(kvc.kvc_attend_workspace_size(c, q, True), dtype=torch.uint8, device=dev)
    got = []
    for x in (q, spoilt):
        out, lse, w = torch.empty_like(q), torch.empty((2, 6, rows), device=dev), torch.full((2, 2, 300), -9.0, device=dev)
        kvc.kvc_attend(c, x, out, lse, weight_out=w, workspace=ws)
        got.append((out, lse, w))
    (o0, l0, w0), (out, lse, w) = got
    assert torch.isnan(out[0, 1, rows - 1]).all() and torch.isnan(lse[0, 1, rows - 1]) and torch.isnan(w[0, 0]).all()
    assert (out[1, 3:] == 0).all() and torch.isneginf(lse[1, 3:]).all()
    out[0, 1, rows - 1], lse[0, 1, rows - 1], w[0, 0] = o0[0, 1, rows - 1], l0[0, 1, rows - 1], w0[0, 0]
    _check_attend(c, q, out, lse, w, torch.zeros_like(w), True, 1 / 8.0)
