"""The decoding operators on the GPU against their definitions in 64 bits (decode_ref.py): rotary positions, the 8-bit cache
(equal code by code), attention over it, eviction, and a run of them together."""
import math

import pytest
import torch

import decode_ref as R
import paper_2509_05165_b200 as kvc
from paper_2509_05165_b200 import workloads as W

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
I8, E4 = torch.int8, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return torch.device("cuda:0")


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _bits(t):
    return t.view(torch.uint8) if t.dtype == E4 else t


# ---- rotary positions --------------------------------------------------------------------------------------------------

ROPES = [
    dict(rot_dim=64), dict(rot_dim=128, interleaved=True, theta=500000.0), dict(rot_dim=32, scaling="linear", factor=4.0),
    dict(rot_dim=128, theta=500000.0, scaling="banded", factor=8.0, turns_low=1.0, turns_high=4.0),
    dict(rot_dim=64, interleaved=True, scaling="yarn", factor=16.0, turns_low=1.0, turns_high=32.0, original_ctx=4096.0),
    dict(rot_dim=16, mscale=0.5), dict(rot_dim=112, interleaved=True),
]


def _rotary_tolerance(x, rope, dtype):
    """A turned pair is off by the angle's error (64 bits in turns up to 2^31 / 2pi: 2^-53 * 2^29 turns, twice, and 2^-25 turns
    where it is cut to fp32, together under 4e-7 rad), sincospif's 2 units (2.4e-7) and three fp32 roundings (1.8e-7): under
    1e-6 of |x1| + |x2|, times m; and half a step of the type."""
    _, m = R.frequencies(rope)
    size = x.double().abs()
    r = rope.rot_dim
    if rope.interleaved:
        size[..., :r] = (size[..., 0:r:2] + size[..., 1:r:2]).repeat_interleave(2, -1)
    else:
        size[..., :r] = (size[..., :r // 2] + size[..., r // 2:r]).repeat(1, 1, 1, 2)
    return 1e-6 * size * max(m, 1.0), torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rope", ROPES, ids=lambda r: "-".join(str(v) for v in r.values()))
@pytest.mark.parametrize("b,hq,hk,rows,far", [(1, 4, 1, 1, 0), (3, 8, 2, 37, 131072), (2, 5, 5, 16, 2 ** 31 - 64), (33, 32, 8, 1, 8192)])
def test_rotary(dev, dtype, rope, b, hq, hk, rows, far):
    rope = kvc.Rotary(**rope)
    for d in (64, 128):
        if rope.rot_dim > d:
            continue
        g = _gen(rows + far)
        q, k = torch.randn((b, hq, rows, d), generator=g).to(dtype), torch.randn((b, hk, rows, d), generator=g).to(dtype)
        pos = torch.randint(0, far + 1, (b, 1), generator=g) + torch.arange(rows)
        qo, ko = torch.full_like(q, 7).to(dev), torch.full_like(k, 7).to(dev)
        kvc.kvc_rotary(rope, q.to(dev), k.to(dev), pos.to(dev), qo, ko)
        for x, y in ((q, qo), (k, ko)):
            want = R.rotate(x, pos, rope)
            tol, half = _rotary_tolerance(x, rope, dtype)
            assert ((y.cpu().double() - want).abs() <= tol + half * (want.abs() + tol)).all()


def test_rotary_in_place_strided_shared_positions_and_back(dev):
    """Heads inside rows (as a projection leaves them), positions for all sequences at once, negative ones, and the inverse,
    which gives the input back (for m = 1) and is the transpose of the forward turn: its gradient."""
    rope, g = kvc.Rotary(64, theta=1e4), _gen(5)
    x = torch.randn((2, 19, 6, 128), generator=g).to(dev)
    q, k = x[:, :, :4].transpose(1, 2), x[:, :, 4:].transpose(1, 2)
    keep = x.clone()
    pos = torch.arange(-9, 10).to(dev)
    want_q = R.rotate(q.cpu(), pos.cpu().expand(2, -1), rope)
    kvc.kvc_rotary(rope, q, k, pos)
    assert (q.cpu().double() - want_q).abs().max() < 2e-5
    kvc.kvc_rotary(rope, q, k, pos, inverse=True)
    assert (x - keep).abs().max() < 2e-5                      # (two turns, each under 1e-6 of values up to 9)
    y, gy = torch.empty_like(q), torch.randn(q.shape, generator=g).to(dev)
    gx = torch.empty_like(q)
    kvc.kvc_rotary(rope, q, None, pos, y)
    kvc.kvc_rotary(rope, gy, None, pos, gx, inverse=True)
    assert abs(float((y.double() * gy.double()).sum() - (q.double() * gx.double()).sum())) < 1e-2   # <Ax, g> = <x, A'g>, 19456 terms
    t = torch.randn(q.shape, generator=g).to(dev)             # and against differences: the turn is linear in x
    a, b_ = torch.empty_like(q), torch.empty_like(q)
    kvc.kvc_rotary(rope, q + 0.5 * t, None, pos, a)
    kvc.kvc_rotary(rope, q - 0.5 * t, None, pos, b_)
    assert abs(float(((a - b_).double() * gy.double()).sum() - (t.double() * gx.double()).sum())) < 1e-2
    only_k = k.contiguous()
    kvc.kvc_rotary(rope, None, only_k, pos)
    assert (only_k.cpu().double() - R.rotate(k.cpu(), pos.cpu().expand(2, -1), rope)).abs().max() < 2e-5


# ---- the 8-bit cache ---------------------------------------------------------------------------------------------------

def _poisoned(b, h, d, cap, block, fmt, dev, lengths=None):
    """A cache whose unused rows hold what must not be read: codes that are no numbers, exponents out of range."""
    c = kvc.alloc_cache(b, h, d, cap, block, fmt, dev)
    for t in (c.k, c.v):
        t.view(torch.uint8).fill_(0x7F)
    c.k_exp.fill_(-128)
    c.v_exp.fill_(127)
    if lengths is not None:
        c.lengths.copy_(lengths.to(torch.int32))
    return c


def _extremes(x):
    """Some rows (and so blocks) of zeros, of the type's smallest and near its largest values, and one at a format's border."""
    if x.shape[-2] > 150:
        x[..., 16:144, :] = 0.0
        x[..., 144:146, :] *= 1e-30
        x[..., 146, :] = 1e-40
    if x.shape[-2] > 300:
        x[..., 290, 3] = 448.0 * 2.0 ** 90
        x[..., 299, 5] = 127.0
    return x


@pytest.mark.parametrize("fmt", [I8, E4])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("d,dtype,per_head,mapped", [(128, BF, False, True), (64, F32, True, True), (128, F32, False, False), (64, BF, True, False)])
def test_gather_into_the_cache(dev, fmt, block, d, dtype, per_head, mapped):
    L, b, h, n, cap = 2, 2, 3, 331, 200
    g = _gen(block)
    k = [_extremes(R.spread_rows(g, b, h, n, d)).to(dtype) for _ in range(L)]
    v = [R.spread_rows(g, b, h, n, d).to(dtype) for _ in range(L)]
    idx = torch.stack([torch.randperm(n, generator=g) for _ in range(L * b * h)]).view(L, b, h, n).to(torch.int32) if mapped else None
    shape = (b, L, h) if per_head else (b, L)
    keep = torch.randint(0, n + 1, shape, generator=g).to(torch.int32)
    keep.view(-1)[0], keep.view(-1)[1] = 0, n                      # none, and more than there is room for
    desc = kvc.kvc_desc_init(L, b, 2 * h, h, d, n, 1, kvc.F32 if dtype == F32 else kvc.BF16)
    caches = [_poisoned(b, h, d, cap, block, fmt, dev) for _ in range(L)]
    clean = [(_bits(c.k).clone(), c.k_exp.clone()) for c in caches]
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    kvc.kvc_cache_gather(desc, [t.to(dev) for t in k], [t.to(dev) for t in v], None if idx is None else idx.to(dev), keep.to(dev), caches,
                         per_head=per_head, device_status=status)
    assert int(status) == -6
    for l, c in enumerate(caches):
        got = R.cache_values(c)
        for i in range(b):
            for j in range(h):
                m = min(cap, int(keep[i, l, j] if per_head else keep[i, l]))
                assert int(c.lengths[i, j]) == m
                rows = idx[l, i, j, :m].long() if mapped else torch.arange(m)
                for t, x in zip((k[l], v[l]), got):
                    want = R.Held(fmt, block).fill(t[i, j][rows]).values(d)
                    assert torch.equal(x[i, j, :m], want)
                assert torch.equal(_bits(c.k)[i, j, m:], clean[l][0][i, j, m:])          # rows behind are left as they were
                assert torch.equal(c.k_exp[i, j, -(-m // block):], clean[l][1][i, j, -(-m // block):])


def test_gather_of_strided_caches_whole_ones_and_bad_positions(dev):
    L, b, h, n, d = 1, 2, 2, 70, 64
    g = _gen(3)
    base = torch.randn((b, n, h, d), generator=g).to(BF).to(dev)              # tokens outside heads
    k = base.transpose(1, 2)
    desc = kvc.kvc_desc_init(L, b, h, h, d, n, 1, kvc.BF16)
    desc.kv_stride[0], desc.kv_stride[1], desc.kv_stride[2] = n * h * d, d, h * d
    store = torch.zeros((b, n + 2, h, d), dtype=I8, device=dev)              # the cache too
    store2 = torch.zeros_like(store)
    exps = lambda: torch.zeros((b, h, 5), dtype=I8, device=dev)  # noqa: E731
    c = kvc.Cache(store.transpose(1, 2), store2.transpose(1, 2), exps(), exps(), torch.zeros((b, h), dtype=torch.int32, device=dev), 16)
    kvc.kvc_cache_gather(desc, [k], [k], None, None, [c])
    assert (c.lengths == n).all()
    want = R.Held(I8, 16).fill(k[1, 0].cpu()).values()
    assert torch.equal(R.cache_values(c)[0][1, 0, :n], want) and torch.equal(R.cache_values(c)[1][1, 0, :n], want)
    idx = torch.arange(n, dtype=torch.int32).expand(1, b, h, n).contiguous()
    idx[..., 5], idx[..., 6], idx[..., 7] = n, -1, 2 ** 31 - 1               # no such tokens: rows of zeros
    kvc.kvc_cache_gather(desc, [k], [k], idx.to(dev), torch.full((b, 1), 40, dtype=torch.int32, device=dev), [c])
    rows = k[0, 1].cpu()[:40].clone()
    rows[5:8] = 0
    assert torch.equal(R.cache_values(c)[0][0, 1, :40], R.Held(I8, 16).fill(rows).values())


@pytest.mark.parametrize("fmt", [I8, E4])
@pytest.mark.parametrize("d,block,dtype,rows", [(128, 64, BF, 1), (64, 16, F32, 1), (128, 128, F32, 3), (128, 16, BF, 100), (64, 128, BF, 300),
                                                (64, 32, F32, 33)])
@pytest.mark.parametrize("in_place", [True, False])
def test_append(dev, fmt, d, block, dtype, rows, in_place):
    h, cap = 2, 400
    have = torch.tensor([0, 1, block - 1, block, block + 1, 3 * block - 1, cap - rows, cap - rows + 1, cap, 7])
    counts = torch.full((10,), rows)
    counts[9] = 0
    b = len(have)
    g = _gen(rows)
    c = _poisoned(b, h, d, cap, block, fmt, dev, have[:, None].expand(-1, h))
    ref = {}
    for i in range(b):
        for j in range(h):
            for name in "kv":
                held = R.Held(fmt, block).fill(0.01 * R.spread_rows(g, int(have[i]), d).to(dtype)) if have[i] else R.Held(fmt, block)
                ref[i, j, name] = held
                for r, (codes, e) in enumerate(zip(held.codes, held.exps)):
                    getattr(c, name)[i, j, r * block:r * block + codes.shape[0]] = codes.float().to(fmt).to(dev)
                    getattr(c, name + "_exp")[i, j, r] = e
    k, v = R.spread_rows(g, b, h, rows, d).to(dtype), R.spread_rows(g, b, h, rows, d).to(dtype)
    k[1], v[1] = 0.0, 1e-6 * v[1]                                             # an open block that does not grow
    weight = torch.full((b, h, cap), 3.0, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    after = None if in_place else torch.full((b, h), -5, dtype=torch.int32, device=dev)
    before = {n: _bits(getattr(c, n)).clone() for n in "kv"}
    kvc.kvc_cache_append(c, k.to(dev), v.to(dev), counts.to(torch.int32).to(dev), after, weight, status)
    assert int(status) == -6
    after = c.lengths if in_place else after
    got = R.cache_values(c)
    for i in range(b):
        new = min(int(counts[i]), cap - int(have[i]))
        n = int(have[i]) + new
        for j in range(h):
            assert int(after[i, j]) == n
            for name, x, src in (("k", got[0], k), ("v", got[1], v)):
                want = ref[i, j, name].append(src[i, j, :new]).values(d)
                assert torch.equal(x[i, j, :n], want), (i, j, name)
                assert torch.equal(_bits(getattr(c, name))[i, j, n:], before[name][i, j, n:])
            w = torch.full((cap,), 3.0)
            w[int(have[i]):n] = 0
            assert torch.equal(weight[i, j].cpu(), w)


@pytest.mark.parametrize("fmt", [I8, E4])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_read(dev, fmt, dtype):
    b, h, d, cap = 2, 2, 64, 90
    c = _poisoned(b, h, d, cap, 32, fmt, dev, torch.tensor([[90, 33], [0, 1]]))
    g = _gen(1)
    vals = [torch.zeros((b, h, cap, d), dtype=torch.float64) for _ in range(2)]
    for i in range(b):
        for j in range(h):
            m = int(c.lengths[i, j])
            for name, x in zip("kv", vals):
                held = R.Held(fmt, 32).fill(R.spread_rows(g, m, d)) if m else R.Held(fmt, 32)
                x[i, j, :m] = held.values(d)
                for r, (codes, e) in enumerate(zip(held.codes, held.exps)):
                    getattr(c, name)[i, j, 32 * r:32 * r + codes.shape[0]] = codes.float().to(fmt).to(dev)
                    getattr(c, name + "_exp")[i, j, r] = e
    for rows, first in ((cap, None), (1, None), (50, torch.tensor([[60, 10], [0, -3]])), (7, torch.tensor([[2 ** 31 - 4, 90], [-2 ** 31, 0]]))):
        f = None if first is None else first.to(torch.int32).to(dev)
        outs = [torch.full((b, h, rows, d), 9.0, dtype=dtype, device=dev) for _ in range(2)]
        kvc.kvc_cache_read(c, outs[0], outs[1], f)
        only = torch.full_like(outs[1], 9.0)
        kvc.kvc_cache_read(c, None, only, f)
        assert torch.equal(only, outs[1])
        for i in range(b):
            for j in range(h):
                f0 = 0 if first is None else int(first[i, j])
                for o, x in zip(outs, vals):
                    want = torch.stack([x[i, j, f0 + r] if 0 <= f0 + r < cap else torch.zeros(d, dtype=torch.float64) for r in range(rows)])
                    assert torch.equal(o[i, j].cpu().double(), want.to(dtype).double())     # exact in bf16 and fp32


# ---- attention ---------------------------------------------------------------------------------------------------------

def _filled_cache(dev, g, b, h, d, cap, block, fmt, lengths, scale_k=1.0, wild=False):
    """Random codes with all their bits in use, exponents that differ from block to block (wild: by up to 2^24)."""
    c = _poisoned(b, h, d, cap, block, fmt, dev, lengths)
    for name in "kv":
        x = torch.randn((b, h, cap, d), generator=g)
        codes = (x * 30).round().clamp(-127, 127).to(I8) if fmt == I8 else (x * 100).clamp(-448, 448).to(E4)
        e = torch.randint(-12, 13, c.k_exp.shape, generator=g) if wild and name == "v" else torch.randint(-1, 2, c.k_exp.shape, generator=g)
        e = e + (round(math.log2(scale_k)) if name == "k" else 0) - (5 if fmt == I8 else 7)
        for i in range(b):
            for j in range(h):
                n = int(lengths[i, j])
                getattr(c, name)[i, j, :n] = codes[i, j, :n].to(dev)
                getattr(c, name + "_exp")[i, j, :-(-n // block)] = e[i, j, :-(-n // block)].to(torch.int8).to(dev)
    return c


def _clean_values(c):
    out = []
    for x in R.cache_values(c):
        live = torch.arange(c.capacity) < c.lengths.cpu()[..., None]
        out.append(torch.where(live[..., None], x, torch.zeros_like(x)))
    return out


def _check_attend(c, q, out, lse, weight, weight0, causal, scale, counts=None):
    """A logit is off by the fp32 sum of d products and the factors on it: under 2^-19 of sum |q k| scale (the products of a
    64-bit sum taken in chunks of 16, each chunk's sum within 2^-22 of its magnitudes) plus 2^-19 for the differences of
    logits of some tens in fp32; a weight p by twice that, relatively (its own and the denominator's).  bf16 outputs: p is
    rounded to 11 bits in front of V and the sum to bf16; fp32: p to 22 bits and the sums of up to thousands of terms, kept in
    fp32 by parts, within 2^-19."""
    k, v = _clean_values(c)
    # P 2^5 (fp32: 2^12) in fp16, relative to a p 2^e of at most the row's largest: numbers below 2^-14 have steps of 2^-24, so p 2^e is
    # off by up to half of 2^-29 (2^-36) of that largest one, for codes of up to 448
    step = torch.pow(torch.tensor(2.0, dtype=torch.float64), c.v_exp.cpu().double()).repeat_interleave(c.block, -1)[..., :c.capacity]
    rel = 2.0 ** -11 if q.dtype == BF else 2.0 ** -19
    o, l, w, mass, size = R.attend(q.cpu().double(), k, v, c.lengths.cpu(), causal, scale, counts, step, 2.0 ** (-29 if q.dtype == BF else -36) / rel)
    dp = 2 * (2.0 ** -19 * size + 2.0 ** -19)
    bf = q.dtype == BF
    got = out.cpu().double()
    rows = torch.ones_like(o, dtype=torch.bool)
    if counts is not None:
        rows = (torch.arange(q.shape[2]) < counts[:, None])[:, None, :, None].expand_as(o)
    tol = (dp + rel) * mass + (2.0 ** -8 if bf else 2.0 ** -23) * o.abs() + 1e-30
    err = ((got - o).abs() - tol)[rows]
    assert torch.isfinite(got[rows]).all() and (err <= 0).all(), float(err.max())
    if lse is not None:
        lr = rows[..., 0]
        g = lse.cpu().double()
        assert torch.equal(torch.isinf(g[lr]), torch.isinf(l[lr]))
        fin = lr & torch.isfinite(l)
        assert ((g - l).abs()[fin] <= dp / 2 + 2.0 ** -22 * l.abs()[fin]).all()
    if weight is not None:
        n = c.lengths.cpu()[..., None]
        live = torch.arange(c.capacity) < n
        want = weight0.cpu().double() + w
        d = (weight.cpu().double() - want).abs()
        assert (d[live] <= (dp * w + 2.0 ** -23 * want)[live] + 1e-30).all(), float(d[live].max())
        assert (weight.cpu()[~live] == -9.0).all()
    return got


ATTEND = [
    # b, h, G, rows, d, block, causal
    (1, 1, 1, 1, 64, 16, True), (2, 2, 4, 1, 128, 64, True), (3, 2, 7, 1, 128, 128, False), (2, 1, 8, 1, 64, 32, True),
    (2, 2, 4, 3, 128, 16, True), (1, 2, 4, 4, 128, 64, False), (2, 1, 2, 17, 64, 64, True), (1, 1, 16, 5, 128, 32, True),
    (1, 1, 3, 50, 128, 128, True), (1, 2, 5, 7, 64, 16, False),
]
LENGTHS = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 250, 511, 513, 900]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("fmt", [I8, E4])
@pytest.mark.parametrize("b,h,G,rows,d,block,causal", ATTEND)
def test_attend(dev, dtype, fmt, b, h, G, rows, d, block, causal):
    g = _gen(rows * 7 + G)
    for turn in range(3):
        lengths = torch.tensor([LENGTHS[int(x)] for x in torch.randint(0, len(LENGTHS), (b * h,), generator=g)]).view(b, h)
        cap = max(1, int(lengths.max())) + (turn * 13)
        c = _filled_cache(dev, g, b, h, d, cap, block, fmt, lengths, wild=turn == 1)
        q = R.spread_rows(g, b, h * G, rows, d).clamp(-8, 8).to(dtype).to(dev)
        out = torch.full_like(q, math.nan)
        lse = torch.full((b, h * G, rows), math.nan, device=dev)
        w0 = torch.rand((b, h, cap), generator=g).to(dev) if turn else None
        weight = torch.full((b, h, cap), -9.0, device=dev) if turn else None
        if turn == 2:                                                        # added to in place
            live = torch.arange(cap, device=dev) < c.lengths[..., None]
            weight = torch.where(live, w0, weight)
        ws = torch.full((kvc.kvc_attend_workspace_size(c, q, turn > 0),), 0xFF, dtype=torch.uint8, device=dev)
        if turn == 2:
            kvc.kvc_attend(c, q, out, lse, weight=weight, causal=causal, workspace=ws)
        else:
            kvc.kvc_attend(c, q, out, lse, weight=w0, weight_out=weight, causal=causal, scale=0.0 if turn else 0.3, workspace=ws)
        _check_attend(c, q, out, lse, weight, w0, causal, 1 / math.sqrt(d) if turn else 0.3)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("fmt", [I8, E4])
def test_attend_over_many_tokens_split_over_the_gpu(dev, dtype, fmt):
    """Few heads, long and very different lengths: parts of a head on many SMs; heads that share an SM with others."""
    g = _gen(11)
    lengths = torch.tensor([[9001, 1], [0, 4096], [130, 20011]])
    c = _filled_cache(dev, g, 3, 2, 128, 20050, 64, fmt, lengths)
    q = torch.randn((3, 8, 2, 128), generator=g).to(dtype).to(dev)
    out, lse = torch.empty_like(q), torch.empty((3, 8, 2), device=dev)
    w0 = torch.zeros((3, 2, 20050), device=dev)
    weight = torch.full_like(w0, -9.0)
    ws = torch.empty(kvc.kvc_attend_workspace_size(c, q, True), dtype=torch.uint8, device=dev)
    kvc.kvc_attend(c, q, out, lse, weight=w0, weight_out=weight, workspace=ws)
    _check_attend(c, q, out, lse, weight, w0, True, 1 / math.sqrt(128))
    again, weight2 = torch.empty_like(out), torch.full_like(w0, -9.0)         # the same bits every time
    for _ in range(3):
        kvc.kvc_attend(c, q, again, weight_out=weight2, workspace=ws)
        assert torch.equal(again, out) and torch.equal(weight2, weight)
    # a sequence's result does not hang on the others of the batch beyond the order of its parts
    one = kvc.Cache(c.k[2:], c.v[2:], c.k_exp[2:], c.v_exp[2:], c.lengths[2:], 64)
    alone = torch.empty_like(q[2:])
    kvc.kvc_attend(one, q[2:], alone, workspace=ws)
    _check_attend(one, q[2:], alone, None, None, None, True, 1 / math.sqrt(128))


def test_attend_padded_batches_strides_and_large_logits(dev):
    g = _gen(4)
    b, h, G, rows, d, cap = 4, 2, 4, 6, 64, 300
    lengths = torch.tensor([[300, 300], [3, 2], [100, 100], [50, 50]])
    c = _filled_cache(dev, g, b, h, d, cap, 32, E4, lengths, scale_k=8.0)
    counts = torch.tensor([6, 5, 0, 1])
    store = torch.randn((b, rows, h * G, d), generator=g).to(BF).to(dev)      # heads inside rows
    q = store.transpose(1, 2)
    ostore = torch.full_like(store, 5.0)
    out = ostore.transpose(1, 2)
    lse = torch.full((b, h * G, rows), 5.0, device=dev)
    weight = torch.full((b, h, cap), -9.0, device=dev)
    ws = torch.empty(kvc.kvc_attend_workspace_size(c, q, True), dtype=torch.uint8, device=dev)
    kvc.kvc_attend(c, q, out, lse, weight_out=weight, row_counts=counts.to(torch.int32).to(dev), workspace=ws)
    _check_attend(c, q, out, lse, weight, torch.zeros_like(weight), True, 1 / 8.0, counts)
    pad = torch.arange(rows) >= counts[:, None]
    assert (ostore.cpu()[pad] == 5.0).all() and (lse.cpu().transpose(1, 2)[pad] == 5.0).all()
    # scores far apart: one token takes all of the softmax
    big = q * 100
    kvc.kvc_attend(c, big, out, lse, row_counts=counts.to(torch.int32).to(dev), workspace=ws)
    k, v = _clean_values(c)
    o = R.attend(big.cpu().double(), k, v, lengths, True, 1 / 8.0, counts)[0]
    got = out.cpu().double()
    live = ~pad[:, None, :, None].expand_as(o)
    # (logits of thousands are off by up to 2^-19 of theirs, so two that lie close may share differently: where one leads by more)
    near = (got - o).abs() <= 0.02 * o.abs() + 0.02 * v.abs().amax()
    assert torch.isfinite(got[live]).all() and near[live].float().mean() > 0.9


def test_attend_queries_and_keys_of_zero_and_tiny_values(dev):
    """All logits equal: the mean of V; queries near the type's smallest; blocks of V of zeros beside large ones."""
    g = _gen(8)
    c = _filled_cache(dev, g, 1, 1, 128, 200, 16, I8, torch.tensor([[200]]))
    c.v[:, :, 32:64] = 0
    c.v_exp[:, :, 2:4] = -100
    for dtype in (BF, F32):
        for s in (0.0, 1e-38, 1e30):
            q = (torch.randn((1, 4, 1, 128), generator=g) * s).to(dtype).to(dev)
            out, lse = torch.empty_like(q), torch.empty((1, 4, 1), device=dev)
            ws = torch.empty(kvc.kvc_attend_workspace_size(c, q, False), dtype=torch.uint8, device=dev)
            kvc.kvc_attend(c, q, out, lse, workspace=ws, scale=1e-30 if s == 1e30 else 0.0)
            _check_attend(c, q, out, lse, None, None, True, 1e-30 if s == 1e30 else 128 ** -0.5)


# ---- eviction ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", [I8, E4])
@pytest.mark.parametrize("d,sb,db,cap,budget,recent", [(128, 64, 64, 700, 300, 100), (64, 16, 128, 333, 64, 0), (128, 128, 32, 700, 128, 128),
                                                      (64, 32, 16, 50, 50, 7), (128, 64, 64, 5000, 1234, 17), (64, 16, 16, 40, 1, 0),
                                                      (64, 16, 16, 40, 1, 1)])
def test_evict(dev, fmt, d, sb, db, cap, budget, recent):
    g = _gen(cap + budget)
    b, h = 3, 2
    lengths = torch.tensor([[cap, cap - 1], [min(budget, cap), min(cap, budget + 1)], [0, max(1, budget // 2)]])
    c = _filled_cache(dev, g, b, h, d, cap, sb, fmt, lengths, wild=True)
    w = torch.rand((b, h, cap), generator=g)
    w[0, 0] = (w[0, 0] * 4).floor()                    # ties
    w[0, 1, ::3] = 0.0
    w[0, 1, ::6] = -0.0
    w[1, 1] = 1.0                                      # all equal
    big = w[..., :].clone()
    dst = _poisoned(b, h, d, budget + 9, db, fmt, dev)
    left = _bits(dst.v).clone()
    idx = torch.full((b, h, budget), -77, dtype=torch.int32, device=dev)
    wo = torch.full((b, h, budget + 9), -9.0, device=dev)
    kvc.kvc_evict(c, dst, big.to(dev), budget, recent, idx, wo)
    k, v = _clean_values(c)
    got = R.cache_values(dst)
    for i in range(b):
        for j in range(h):
            kept = R.evict(w[i, j], int(lengths[i, j]), budget, recent)
            m = len(kept)
            assert int(dst.lengths[i, j]) == m
            assert idx[i, j].tolist() == kept + [-1] * (budget - m)
            assert torch.equal(wo[i, j, :m].cpu(), w[i, j][kept]) and (wo[i, j, m:] == -9.0).all()
            for x, y in zip((k, v), got):
                assert torch.equal(y[i, j, :m], R.Held(fmt, db).fill(x[i, j][kept]).values(d))
            assert torch.equal(_bits(dst.v)[i, j, m:], left[i, j, m:])


@pytest.mark.parametrize("n,budget,recent,h", [(60001, 20011, 333, 2), (350003, 9000, 0, 1), (350003, 340000, 200000, 1), (9000, 8999, 1, 3)])
def test_evict_from_long_rows(dev, n, budget, recent, h):
    """Rows shared by up to eight CTAs, and longer than these keep; ties over all of them, negative and infinite weights."""
    g = _gen(n)
    c = kvc.alloc_cache(1, h, 64, n + 3, 64, I8, dev)
    c.k.random_(-100, 100)
    c.lengths.fill_(n)
    w = torch.randn((1, h, n + 3), generator=g).exp()
    w[0, 0] = (w[0, 0] * 2).floor()                    # few values, many ties
    if h > 1:
        w[0, 1, ::5] *= -1.0
        w[0, 1, 17], w[0, 1, 18] = math.inf, -math.inf
    dst = kvc.alloc_cache(1, h, 64, budget, 64, I8, dev)
    idx, wo = torch.empty((1, h, budget), dtype=torch.int32, device=dev), torch.empty((1, h, budget), device=dev)
    kvc.kvc_evict(c, dst, w.to(dev), budget, recent, idx, wo)
    free = n - recent
    for j in range(h):
        heavy = torch.sort(w[0, j, :free], descending=True, stable=True).indices[:budget - recent].sort().values
        kept = torch.cat([heavy, torch.arange(free, n)])
        assert torch.equal(idx[0, j].cpu().long(), kept) and torch.equal(wo[0, j].cpu(), w[0, j][kept])
        a, b = c.k[0, j][kept.to(dev)].float() * torch.pow(2.0, c.k_exp[0, j][kept.to(dev) // 64].float())[:, None], None
        b = dst.k[0, j].float() * torch.pow(2.0, dst.k_exp[0, j].float()).repeat_interleave(64)[:budget, None]
        assert torch.equal(a, b)                       # (codes of up to 100 under one exponent keep their values)


# ---- what the calls allow beyond the ordinary --------------------------------------------------------------------------

def test_host_tensors_are_refused_beside_a_gpu(dev):
    c = kvc.alloc_cache(1, 1, 64, 20, 16, I8, "cpu")
    q = torch.zeros((1, 1, 1, 64), dtype=BF)
    ws = torch.zeros(kvc.kvc_attend_workspace_size(c, q, False) + 256, dtype=torch.uint8)
    for call in (lambda: kvc.kvc_attend(c, q, q.clone(), workspace=ws[-ws.data_ptr() % 256:]), lambda: kvc.kvc_cache_append(c, q, q),
                 lambda: kvc.kvc_cache_read(c, q, None), lambda: kvc.kvc_rotary(kvc.Rotary(64), q, None, torch.zeros(1, dtype=torch.int64)),
                 lambda: kvc.kvc_attend(kvc.alloc_cache(1, 1, 64, 20, 16, I8, dev), q.to(dev), q, workspace=ws.to(dev))):
        with pytest.raises(kvc.KvcError) as e:
            call()
        assert e.value.status == -1


def test_gather_into_caches_of_different_capacities(dev):
    """Layers keep different numbers of rows, so their caches differ; with and without room to spare."""
    L, h, d, n = 3, 2, 64, 260
    g = _gen(21)
    k, v = [[torch.randn((1, h, n, d), generator=g).to(BF).to(dev) for _ in range(L)] for _ in range(2)]
    keep = torch.tensor([[7, 260, 129]], dtype=torch.int32)
    caches = [_poisoned(1, h, d, cap, 32, E4, dev) for cap in (7, 300, 130)]
    desc = kvc.kvc_desc_init(L, 1, h, h, d, n, 1, kvc.BF16)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    kvc.kvc_cache_gather(desc, k, v, None, keep.to(dev), caches, device_status=status)
    assert int(status) == 0
    for l, c in enumerate(caches):
        m = int(keep[0, l])
        assert (c.lengths == m).all()
        for x, src in zip(R.cache_values(c), (k, v)):
            for j in range(h):
                assert torch.equal(x[0, j, :m], R.Held(E4, 32).fill(src[l][0, j, :m].cpu()).values())


@pytest.mark.parametrize("fmt", [I8, E4])
def test_heads_inside_tokens_and_offsets_beyond_32_bits(dev, fmt):
    """A cache whose second sequence, or whose tokens, lie gigabytes apart, and rows as a projection leaves them: the same as a
    dense one, code by code and bit by bit."""
    g = _gen(31)
    b, h, d, cap, rows = 2, 2, 64, 70, 40
    k_new, v_new = [R.spread_rows(g, b, rows, h, d).to(BF).to(dev).transpose(1, 2) for _ in range(2)]
    q = torch.randn((b, 3, 2 * h, d), generator=g).to(BF).to(dev).transpose(1, 2)
    big = 2 ** 32 + 2 ** 20
    for stride in ((big, d, h * d, 1), (d * h, d, big // 64 // 16 * 16, 1)):
        span = sum((s - 1) * t for s, t in zip((b, h, cap), stride)) + d
        stores = [torch.empty(span, dtype=torch.uint8, device=dev) for _ in range(2)]
        views = [s.view(fmt).as_strided((b, h, cap, d), stride) for s in stores]
        dense = kvc.alloc_cache(b, h, d, cap, 16, fmt, dev)
        far = kvc.Cache(*views, torch.zeros_like(dense.k_exp), torch.zeros_like(dense.v_exp), torch.zeros_like(dense.lengths), 16)
        outs = []
        for c in (dense, far):
            kvc.kvc_cache_append(c, k_new, v_new)
            kvc.kvc_cache_append(c, k_new[:, :, :25], v_new[:, :, :25])
            out, lse = torch.empty_like(q), torch.empty((b, 2 * h, 3), device=dev)
            weight = torch.zeros((b, h, cap), device=dev)
            ws = torch.empty(kvc.kvc_attend_workspace_size(c, q, True), dtype=torch.uint8, device=dev)
            kvc.kvc_attend(c, q, out, lse, weight=weight, workspace=ws)
            ko, vo = [torch.empty((b, h, cap, d), dtype=F32, device=dev) for _ in range(2)]
            kvc.kvc_cache_read(c, ko, vo)
            small = kvc.alloc_cache(b, h, d, 30, 32, fmt, dev)
            idx = torch.empty((b, h, 30), dtype=torch.int32, device=dev)
            kvc.kvc_evict(c, small, weight, 30, 8, idx)
            outs.append([c.lengths, c.k_exp, c.v_exp, out, lse, weight, ko, vo, idx, _bits(small.k), small.v_exp])
        assert all(torch.equal(x, y) for x, y in zip(*outs))
        assert (outs[0][0] == 65).all()
        want = torch.cat([R.Held(fmt, 16).append(k_new[1, 1].cpu()).append(k_new[1, 1, :25].cpu()).values(), torch.zeros((5, d))])
        assert torch.equal(outs[0][6][1, 1].cpu().double(), want)
        del stores, views, far, outs
        torch.cuda.empty_cache()


def test_many_query_heads_and_rows_of_one_head(dev):
    """More query rows of a KV head than one launch takes, with weights; and the same call captured twice over one workspace."""
    g = _gen(41)
    lengths = torch.tensor([[333], [50]])
    c = _filled_cache(dev, g, 2, 1, 64, 340, 64, I8, lengths)
    q = torch.randn((2, 128, 2, 64), generator=g).to(BF).to(dev)
    out, lse = torch.empty_like(q), torch.empty((2, 128, 2), device=dev)
    w0 = torch.rand((2, 1, 340), generator=g).to(dev)
    weight = torch.full_like(w0, -9.0)
    ws = torch.empty(kvc.kvc_attend_workspace_size(c, q, True), dtype=torch.uint8, device=dev)
    kvc.kvc_attend(c, q, out, lse, weight=w0, weight_out=weight, workspace=ws)
    _check_attend(c, q, out, lse, weight, w0, True, 1 / 8.0)
    few, small = q[:, :2].contiguous(), torch.empty_like(q[:, :2])
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0]):
        kvc.kvc_attend(c, q, out, workspace=ws)
    with torch.cuda.graph(graphs[1]):
        kvc.kvc_attend(c, few, small, workspace=ws)
    want, want_small = out.clone(), torch.empty_like(small)
    kvc.kvc_attend(c, few, want_small, workspace=ws)
    for _ in range(3):
        out.zero_()
        small.zero_()
        graphs[0].replay()
        graphs[1].replay()
        assert torch.equal(out, want) and torch.equal(small, want_small)


@pytest.mark.parametrize("rows", [1, 5])
def test_more_heads_than_threads(dev, rows):
    """1400 heads, most of them empty or of a few tokens, some long: every warp holds several of them; and their eviction."""
    g = _gen(51 + rows)
    b, h, d, cap = 700, 2, 64, 700
    lengths = torch.randint(0, 40, (b, h), generator=g)
    lengths[torch.rand((b, h), generator=g) < 0.4] = 0
    lengths[::97, 1] = torch.randint(100, cap + 1, (len(lengths[::97]),), generator=g)
    k, v = [torch.randint(-127, 128, (b, h, cap, d), generator=g).to(I8) for _ in range(2)]
    ke, ve = [torch.randint(-9, -5, (b, h, -(-cap // 128)), generator=g).to(I8) for _ in range(2)]
    c = kvc.Cache(k.to(dev), v.to(dev), ke.to(dev), ve.to(dev), lengths.to(torch.int32).to(dev), 128)
    q = torch.randn((b, 3 * h, rows, d), generator=g).to(BF).to(dev)
    out, lse = torch.empty_like(q), torch.empty((b, 3 * h, rows), device=dev)
    w0 = torch.rand((b, h, cap), generator=g).to(dev)
    weight = torch.full_like(w0, -9.0)
    ws = torch.full((kvc.kvc_attend_workspace_size(c, q, True),), 0xFF, dtype=torch.uint8, device=dev)
    kvc.kvc_attend(c, q, out, lse, weight=w0, weight_out=weight, workspace=ws)
    _check_attend(c, q, out, lse, weight, w0, True, 1 / 8.0)
    dst = kvc.alloc_cache(b, h, d, 20, 16, I8, dev)
    idx = torch.empty((b, h, 20), dtype=torch.int32, device=dev)
    kvc.kvc_evict(c, dst, weight, 20, 3, idx)
    w, got = weight.cpu(), idx.cpu()
    for i in range(b):
        for j in range(h):
            kept = R.evict(w[i, j], int(lengths[i, j]), 20, 3)
            assert got[i, j].tolist() == kept + [-1] * (20 - len(kept))


def test_calls_at_once_on_two_streams_and_captured_moves(dev):
    """Calls that share nothing but the cache they read, in flight together; and append, eviction and reading in a graph."""
    g = _gen(61)
    c = _filled_cache(dev, g, 2, 2, 128, 6000, 64, E4, torch.tensor([[6000, 5000], [77, 0]]))
    q = torch.randn((2, 8, 1, 128), generator=g).to(BF).to(dev)
    w = torch.rand((2, 2, 6000), generator=g).to(dev)
    ws = [torch.empty(kvc.kvc_attend_workspace_size(c, q, True), dtype=torch.uint8, device=dev) for _ in range(3)]
    want, want_w = torch.empty_like(q), torch.full_like(w, -9.0)
    kvc.kvc_attend(c, q, want, weight=w, weight_out=want_w, workspace=ws[2])
    outs, sums = [torch.empty_like(q) for _ in range(2)], [torch.full_like(w, -9.0) for _ in range(2)]
    streams = [torch.cuda.Stream(dev) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, o, x, y in zip(streams, outs, sums, ws):
            kvc.kvc_attend(c, q, o, weight=w, weight_out=x, workspace=y, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) and torch.equal(x, want_w) for o, x in zip(outs, sums))
    spare, idx = kvc.alloc_cache(2, 2, 128, 600, 32, E4, dev), torch.empty((2, 2, 500), dtype=torch.int32, device=dev)
    k_new = torch.randn((2, 2, 9, 128), generator=g).to(BF).to(dev)
    back = torch.empty((2, 2, 600, 128), dtype=BF, device=dev)

    def moves():
        kvc.kvc_evict(c, spare, w, 500, 100, idx)
        kvc.kvc_cache_append(spare, k_new, k_new)
        kvc.kvc_cache_read(spare, back, None)

    moves()
    plain = [t.clone() for t in (back, idx, spare.lengths, _bits(spare.v))]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moves()
    for _ in range(2):
        spare.k.view(torch.uint8).fill_(0x7F)
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(plain[:3], (back, idx, spare.lengths)))


# ---- together ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt,dtype", [(E4, BF), (I8, F32)])
def test_compress_then_decode(dev, fmt, dtype):
    """A prompt's cache is compressed and held in 8 bits; tokens are rotated, appended and attended with, in a captured and
    replayed step on a stream of its own; then the cache is cut back by what its tokens were worth."""
    L, hq, h, d, n, block, steps = 2, 8, 2, 64, 500, 16, 20
    cfg = W.WorkloadConfig("decode", L, hq, h, d, n, 16, batch=2, dtype="f32" if dtype == F32 else "bf16", retention=0.3, elem_std=1.0)
    wl = W.make_workload(cfg, dev)
    desc = kvc.desc_from_config(cfg, keep_position_order=1)
    out = kvc.compress(wl.q, wl.k, wl.v, desc, cfg.budget)
    cap = int(out.n_keep.max()) + steps
    caches = [kvc.alloc_cache(2, h, d, cap, block, fmt, dev) for _ in range(L)]
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    kvc.kvc_cache_gather(desc, wl.k, wl.v, out.idx, out.n_keep, caches, device_status=status)
    keep, off = out.n_keep.cpu(), out.offsets.cpu()
    held = {}
    for l in range(L):
        for i in range(2):
            kl, vl = out.layer(i, l, keep, off, h, d)                     # K', V' as kvc_gather writes them: the same rows
            for j in range(h):
                held[l, i, j] = [R.Held(fmt, block).fill(x[j].cpu()) for x in (kl, vl)]
    g = _gen(2)
    rope = kvc.Rotary(64, theta=1e4)
    tokens = [[torch.randn((2, m, 1, d), generator=g).to(dtype) for m in (hq, h, h)] for _ in range(steps * L)]
    weights = [torch.zeros((2, h, cap), device=dev) for _ in range(L)]
    q, k, v = (torch.zeros_like(t).to(dev) for t in tokens[0])
    pos = torch.zeros((2, 1), dtype=torch.int64, device=dev)
    o = torch.empty_like(q)
    ws = torch.empty(kvc.kvc_attend_workspace_size(caches[0], q, True), dtype=torch.uint8, device=dev)

    def step(l):
        kvc.kvc_rotary(rope, q, k, pos)
        kvc.kvc_cache_append(caches[l], k, v, weight=weights[l], device_status=status)
        kvc.kvc_attend(caches[l], q, o, weight=weights[l], workspace=ws)

    side = torch.cuda.Stream(dev)
    graphs = []
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for l in range(L):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step(l)
            graphs.append(graph)
        want_w = [torch.zeros((2, h, cap), dtype=torch.float64) for _ in range(L)]
        for t in range(steps):
            for l in range(L):
                for x, y in zip((q, k, v), tokens[t * L + l]):
                    x.copy_(y)
                pos.fill_(n + t)
                graphs[l].replay()
                side.synchronize()
                tq, tk, tv = tokens[t * L + l]
                rq, rk = R.rotate(tq, torch.full((2, 1), n + t), rope), k.cpu()
                assert (rk.double() - R.rotate(tk, torch.full((2, 1), n + t), rope)).abs().max() < (0.04 if dtype == BF else 1e-5)
                vals = [torch.zeros((2, h, cap, d), dtype=torch.float64) for _ in range(2)]
                for i in range(2):
                    for j in range(h):
                        m = 0
                        for x, dst, src in zip(held[l, i, j], vals, (rk, tv)):
                            x.append(src[i, j])
                            m = x.values(d).shape[0]
                            dst[i, j, :m] = x.values(d)
                        assert int(caches[l].lengths[i, j]) == m
                got = _clean_values(caches[l])
                assert torch.equal(got[0], vals[0]) and torch.equal(got[1], vals[1])
                want, _, w, mass, size = R.attend(q.cpu().double(), vals[0], vals[1], caches[l].lengths.cpu(), True, d ** -0.5)
                want_w[l] += w
                assert (q.cpu().double() - rq).abs().max() < (0.04 if dtype == BF else 1e-5)
                tol = 2.0 ** -8 * want.abs() + 2.0 ** -10 * mass if dtype == BF else 2e-4 * mass
                assert ((o.cpu().double() - want).abs() <= tol + 1e-6).all()
    assert int(status) == 0
    for l in range(L):
        assert (weights[l].cpu().double() - want_w[l]).abs().max() < 1e-4 * steps
        spare = kvc.alloc_cache(2, h, d, 64, block, fmt, dev)
        idx = torch.empty((2, h, 48), dtype=torch.int32, device=dev)
        kvc.kvc_evict(caches[l], spare, weights[l], 48, 10, idx)
        got = R.cache_values(spare)
        for i in range(2):
            for j in range(h):
                m = int(caches[l].lengths[i, j])
                kept = R.evict(weights[l][i, j].cpu(), m, 48, 10)
                assert idx[i, j].tolist() == kept + [-1] * (48 - len(kept))
                for x, y in zip(held[l, i, j], got):
                    assert torch.equal(y[i, j, :len(kept)], R.Held(fmt, block).fill(x.values(d)[kept]).values(d))
