"""The operators of decoding from a compressed cache, through the package's public entry points, and in plain torch.

A case names one operator (`kind`) and its shape:
  rotary   `kvc_rotary`: rotary positions of queries and keys, before they are scored, cached or attended with
  gather   `kvc_cache_gather` + `kvc_cache_read`: the kept rows of a prefilled cache into an 8-bit one, and its values
  append   `kvc_cache_append` + `kvc_cache_read`: the rows of new tokens into the open blocks of an 8-bit cache, and the
           values of the blocks that this touched
  attend   `kvc_attend`: attention of a few query rows over an 8-bit cache, with the tokens' running weight
  evict    `kvc_evict` + `kvc_cache_read`: the heaviest and the latest tokens of an 8-bit cache into another, its values

The 8-bit cache: `block` tokens of a head share one exponent, K and V apart.  With amax the block's largest magnitude, the
exponent e is the smallest whole number with amax <= qmax 2^e (qmax 127 for int8, 448 for e4m3), within [-100, 121]; a code
is the value times 2^-e, rounded to nearest, ties to even, and it stands for code 2^e.
"""
import math

import torch

own = False

_FORMATS = {"int8": (127.0, torch.int8), "e4m3": (448.0, torch.float8_e4m3fn)}
_E_MIN, _E_MAX = -100, 121

_BASE = dict(q_heads=32, kv_heads=8, head_dim=128, batch=1, dtype="bf16", fmt="e4m3", block=64)


def _case(kind, **kw):
    return dict(_BASE, kind=kind, **kw)


def listed():
    return [
        # one decoding step of a serving batch: queries and keys of one token each, positions far into the context
        _case("rotary", name="rotary_step_32", batch=32, rows=1, layout="half", rot_dim=128, scaling="banded", far=131072),
        # a prompt of an odd length, the 8B shape
        _case("rotary", name="rotary_prompt_16k", rows=16001, layout="half", rot_dim=128, scaling="banded", far=0),
        # the 8B shape at 8K with a quarter kept, all layers in one call
        _case("gather", name="gather_8b_8k", layers=32, n_ctx=8192, keep=2048, per_head=False, idx=True),
        # a small fp32 cache of an odd length, every head with its own tokens
        _case("gather", name="gather_f32_odd", layers=4, batch=2, q_heads=4, kv_heads=2, head_dim=64, n_ctx=1001, keep=333,
              dtype="f32", fmt="int8", block=32, per_head=True, idx=True),
        # one token of every sequence of a serving batch
        _case("append", name="append_step_32", batch=32, capacity=4096, rows=1),
        # a turn of 500 tokens per sequence behind caches of different lengths
        _case("append", name="append_turn_500", batch=8, capacity=4096, rows=500, fmt="int8", block=32),
        # a short context: latency
        _case("attend", name="attend_1k", length=1000, rows=1, ragged=False, weights=False, causal=True),
        # the 8B shape over the whole of 32K tokens, the tokens' weight kept
        _case("attend", name="attend_32k_weights", length=32768, rows=1, ragged=False, weights=True, causal=True),
        # a serving batch of very different lengths (some empty), int8
        _case("attend", name="attend_batch_ragged", batch=32, length=16384, rows=1, ragged=True, weights=True, causal=True,
              fmt="int8", block=32),
        # the long-context shape, four rows at once (drafted tokens)
        _case("attend", name="attend_128k_rows4", q_heads=28, kv_heads=4, length=131072, rows=4, ragged=False, weights=False,
              causal=True, block=128),
        # all layers of the 8B shape back to 2048 tokens after 64 more
        _case("evict", name="evict_64_of_2112", batch=32, length=2112, budget=2048, recent=512, ragged=False),
        # long sequences of different lengths down to a quarter, int8
        _case("evict", name="evict_batch_32k", batch=8, length=32768, budget=8192, recent=1001, ragged=True, fmt="int8", block=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "gather", "append", "attend", "attend", "evict"])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    head_dim = rng.choice([64, 128, 128])
    c = dict(kv_heads=kv_heads, q_heads=kv_heads * rng.choice([1, 2, 4, 4, 7, 8]), head_dim=head_dim,
             dtype="f32" if rng.random() < 0.2 else "bf16", fmt=rng.choice(["e4m3", "int8"]), block=rng.choice([16, 32, 64, 128]),
             batch=_log_int(rng, 1, 32))
    if kind == "rotary":
        tokens = _log_int(rng, 1, 16001)        # (no more than the listed prompt, in rows of all sequences together)
        c.update(batch=min(c["batch"], tokens), layout=rng.choice(["half", "interleaved"]),
                 rot_dim=rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4]),
                 scaling=rng.choice(["none", "linear", "banded", "yarn"]), far=rng.choice([0, 0, 131072, 2 ** 30]))
        heads = (c["q_heads"] + kv_heads) * (2 if c["dtype"] == "f32" else 1) * head_dim
        c["rows"] = max(1, min(tokens // c["batch"], 16001 * 40 * 128 // (heads * c["batch"])))
        return _case(kind, **c)
    if kind == "gather":
        layers, c["batch"] = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([1, 1, 2, 4])
        most = 32 * 8192 * 8 * 128 // (layers * c["batch"] * kv_heads * head_dim * (2 if c["dtype"] == "f32" else 1))
        n = _log_int(rng, 64, min(32768, most))
        c.update(layers=layers, n_ctx=n, keep=min(max(1, int(n * rng.uniform(0.02, 0.5))), most // 4),
                 per_head=rng.random() < 0.4, idx=rng.random() < 0.8)
        return _case(kind, **c)
    if kind == "append":
        c["rows"] = 1 if rng.random() < 0.5 else _log_int(rng, 2, 500)
        c["batch"] = max(1, min(c["batch"], 8 if c["rows"] > 1 else 32))
        if c["dtype"] == "f32":
            c["batch"] = max(1, c["batch"] // 2)
        c["capacity"] = c["rows"] + _log_int(rng, 1, 4096)
        return _case(kind, **c)
    if kind == "attend":
        c["rows"] = 1 if rng.random() < 0.6 else rng.randint(2, 16)
        # tokens of all sequences and heads, bounded by codes read and by products
        most = 32 * 8 * 16384 * 128 // 4 // (c["batch"] * kv_heads * head_dim)
        if c["rows"] > 1:
            most = min(most, 28 * 4 * 131072 * 128 // (c["rows"] * c["batch"] * c["q_heads"] * head_dim))
        c.update(length=_log_int(rng, 1, max(1, min(131072, most))), ragged=rng.random() < 0.5, weights=rng.random() < 0.5,
                 causal=rng.random() < 0.7)
        return _case(kind, **c)
    most = 8 * 8 * 32768 * 128 // (c["batch"] * kv_heads * head_dim)
    n = _log_int(rng, 16, min(65536, most))
    budget = max(1, min(int(n * rng.uniform(0.1, 1.0)), 8 * 8 * 8192 * 128 // (c["batch"] * kv_heads * head_dim)))
    c.update(dtype="bf16", length=n, budget=budget, recent=int(budget * rng.choice([0.0, 0.25, 0.5, 1.0])), ragged=rng.random() < 0.5)
    return _case(kind, **c)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _keys_values(shape, queries, gen, dev):
    """Rows [..., n, d] of keys and values: channels of different size, a few keys along the mean query, as prompts give."""
    d = shape[-1]
    ch = torch.exp(0.5 * torch.randn((d,), generator=gen, device=dev))
    k = torch.randn(shape, generator=gen, device=dev) * ch
    heavy = torch.rand(shape[:-1] + (1,), generator=gen, device=dev) < 0.01
    k = torch.where(heavy, k + 2.0 * queries, k)
    # value rows of different lengths
    v = torch.randn(shape, generator=gen, device=dev) * torch.exp(torch.randn(shape[:-1] + (1,), generator=gen, device=dev))
    return k, v


def _filled(c, n, gen, dev):
    """A cache of `n` rows per head, every one of them written, in a cache with room for some more."""
    cap = n + 5
    q = torch.randn((c["batch"], c["kv_heads"], 1, c["head_dim"]), generator=gen, device=dev)
    k, v = _keys_values((c["batch"], c["kv_heads"], cap, c["head_dim"]), q, gen, dev)
    kc, ke = _quantise(k, c["fmt"], c["block"])
    vc, ve = _quantise(v, c["fmt"], c["block"])
    return dict(k=kc, v=vc, k_exp=ke, v_exp=ve), q


def _lengths(c, n, gen, dev):
    """Lengths [batch, heads]; ragged: one per sequence, spread over their logarithm, the first `n` and the second empty."""
    if not c["ragged"]:
        return torch.full((c["batch"], c["kv_heads"]), n, dtype=torch.int32, device=dev)
    t = torch.exp(torch.rand((c["batch"],), generator=gen, device=dev) * math.log(n + 1.0)).long().clamp_(1, n)
    t[0] = n
    t[1:2] = 0
    return t.to(torch.int32)[:, None].expand(-1, c["kv_heads"]).contiguous()


def _empty_cache(c, batch, cap, dev):
    codes = torch.zeros((batch, c["kv_heads"], cap, c["head_dim"]), dtype=_FORMATS[c["fmt"]][1], device=dev)
    exps = torch.zeros((batch, c["kv_heads"], -(-cap // c["block"])), dtype=torch.int8, device=dev)
    return dict(k=codes, v=codes.clone(), k_exp=exps, v_exp=exps.clone(),
                lengths=torch.zeros((batch, c["kv_heads"]), dtype=torch.int32, device=dev))


def prepare(case, seed):
    c = dict(_BASE, **case)
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt, d, b, h = _dtype(c), c["head_dim"], c["batch"], c["kv_heads"]
    st = dict(c=c)
    if c["kind"] == "rotary":
        st["q"] = torch.randn((b, c["q_heads"], c["rows"], d), generator=gen, device=dev).to(dt)
        st["k"] = torch.randn((b, h, c["rows"], d), generator=gen, device=dev).to(dt)
        first = torch.randint(0, c["far"] + 1, (b, 1), generator=gen, device=dev)
        st["positions"] = first + torch.arange(c["rows"], device=dev)
        st["q_out"], st["k_out"] = torch.empty_like(st["q"]), torch.empty_like(st["k"])
    elif c["kind"] == "gather":
        shape = (c["layers"], b, h, c["n_ctx"], d)
        k, v = torch.empty(shape, dtype=dt, device=dev), torch.empty(shape, dtype=dt, device=dev)
        for layer in range(c["layers"]):
            q = torch.randn((b, h, 1, d), generator=gen, device=dev)
            kl, vl = _keys_values(shape[1:], q, gen, dev)
            k[layer], v[layer] = kl, vl
        st["k"], st["v"] = k, v
        # a ranking per head, and a number of kept rows per layer (or head) that sums to about a share of them
        st["idx"] = torch.rand(shape[:-1], generator=gen, device=dev).argsort(-1).to(torch.int32) if c["idx"] else None
        rows = (b, c["layers"], h) if c["per_head"] else (b, c["layers"])
        st["n_keep"] = (torch.rand(rows, generator=gen, device=dev) * (c["keep"] + 1)).long().clamp_(0, c["keep"]).to(torch.int32)
        st["cache"] = _empty_cache(c, c["layers"] * b, c["keep"], dev)
        st["k_out"] = torch.empty((c["layers"] * b, h, c["keep"], d), dtype=dt, device=dev)
        st["v_out"] = torch.empty_like(st["k_out"])
    elif c["kind"] == "append":
        st["cache"], q = _filled(c, c["capacity"], gen, dev)
        st["cache"]["lengths"] = torch.randint(0, c["capacity"] - c["rows"] + 1, (b, 1), generator=gen, device=dev,
                                               dtype=torch.int32).expand(-1, h).contiguous()
        k, v = _keys_values((b, h, c["rows"], d), q, gen, dev)
        st["k_new"], st["v_new"] = k.to(dt), v.to(dt)
        st["lengths_out"] = torch.empty_like(st["cache"]["lengths"])
        st["first"] = st["cache"]["lengths"] // c["block"] * c["block"]
        st["k_out"] = torch.empty((b, h, c["rows"] + c["block"], d), dtype=dt, device=dev)
        st["v_out"] = torch.empty_like(st["k_out"])
    elif c["kind"] == "attend":
        st["cache"], q = _filled(c, c["length"], gen, dev)
        st["cache"]["lengths"] = _lengths(c, c["length"], gen, dev)
        group = c["q_heads"] // h
        noise = torch.randn((b, h, group * c["rows"], d), generator=gen, device=dev)
        st["q"] = (q + noise).reshape(b, c["q_heads"], c["rows"], d).to(dt)
        st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty((b, c["q_heads"], c["rows"]), device=dev)
        if c["weights"]:
            st["weight"] = torch.rand((b, h, c["length"] + 5), generator=gen, device=dev)
            st["weight_out"] = torch.zeros_like(st["weight"])
    else:
        st["cache"], _ = _filled(c, c["length"], gen, dev)
        st["cache"]["lengths"] = _lengths(c, c["length"], gen, dev)
        # accumulated weights: a few heavy tokens, many light ones, some of them equal
        w = torch.exp(2.0 * torch.randn((b, h, c["length"] + 5), generator=gen, device=dev))
        st["weight"] = torch.where(w < 0.2, torch.zeros_like(w), w)
        st["dst"] = _empty_cache(c, b, c["budget"], dev)
        st["idx"] = torch.empty((b, h, c["budget"]), dtype=torch.int32, device=dev)
        st["weight_out"] = torch.zeros((b, h, c["budget"]), device=dev)
        st["k_out"] = torch.empty((b, h, c["budget"], d), dtype=dt, device=dev)
        st["v_out"] = torch.empty_like(st["k_out"])
    return st


# ---- the plain forms ------------------------------------------------------------------------------------------------

_THETA, _FACTOR, _ORIGINAL = 500000.0, 8.0, 8192.0
_TURNS = {"banded": (1.0, 4.0), "yarn": (1.0, 32.0)}


def _frequencies(c, dev):
    """Angle per position of each pair, in 64 bits, and the factor on the rotated values."""
    i = torch.arange(c["rot_dim"] // 2, device=dev, dtype=torch.float64)
    f = _THETA ** (-2.0 * i / c["rot_dim"])
    if c["scaling"] == "linear":
        return f / _FACTOR, 1.0
    if c["scaling"] == "banded":
        lo, hi = _TURNS["banded"]
        turns = _ORIGINAL * f / (2.0 * math.pi)
        keep = ((turns - lo) / (hi - lo)).clamp(0.0, 1.0)
        return keep * f + (1.0 - keep) * f / _FACTOR, 1.0
    if c["scaling"] == "yarn":
        lo, hi = _TURNS["yarn"]
        first = max(0, math.floor(c["rot_dim"] * math.log(_ORIGINAL / (hi * 2.0 * math.pi)) / (2.0 * math.log(_THETA))))
        last = min(c["rot_dim"] - 1, math.ceil(c["rot_dim"] * math.log(_ORIGINAL / (lo * 2.0 * math.pi)) / (2.0 * math.log(_THETA))))
        ramp = ((i - first) / max(last - first, 0.001)).clamp(0.0, 1.0)
        return (1.0 - ramp) * f + ramp * f / _FACTOR, 0.1 * math.log(_FACTOR) + 1.0
    return f, 1.0


def _rotate(x, cos, sin, c):
    y, rot = x.float(), c["rot_dim"]
    if c["layout"] == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _plain_rotary(st):
    c = st["c"]
    f, factor = _frequencies(c, st["q"].device)
    angle = st["positions"].double()[:, None, :, None] * f
    cos, sin = (torch.cos(angle) * factor).float(), (torch.sin(angle) * factor).float()
    return [_rotate(st["q"], cos, sin, c), _rotate(st["k"], cos, sin, c)]


def _exponent(amax, fmt):
    """The smallest e with amax <= qmax 2^e, exactly."""
    m, e = torch.frexp(amax)                    # amax = m 2^e, m in [1/2, 1)
    qm, qe = math.frexp(_FORMATS[fmt][0])
    return (e - qe + (m > qm).to(e.dtype)).masked_fill(amax == 0, _E_MIN).clamp(_E_MIN, _E_MAX)


def _pow2(e):
    """2^e, exactly, of whole numbers (a power function need not be exact, and ties would then round the wrong way)."""
    return ((e.int().clamp(-126, 127) + 127) << 23).view(torch.float32)


def _code(x, e, fmt):
    """x 2^-e rounded to the format, as the format's values in fp32."""
    y = x.float() * _pow2(-e)
    return torch.round(y) if fmt == "int8" else y.to(torch.float8_e4m3fn).float()


def _blocks(x, block, n):
    """[..., n, d] as [..., blocks, block, d], rows behind the last one zero."""
    pad = -n % block
    x = torch.cat([x, x.new_zeros(x.shape[:-2] + (pad, x.shape[-1]))], -2) if pad else x
    return x.unflatten(-2, (-1, block))


def _quantise(x, fmt, block):
    n = x.shape[-2]
    y = _blocks(x.float(), block, n)
    e = _exponent(y.abs().amax((-1, -2)), fmt)
    codes = _code(y, e[..., None, None], fmt).flatten(-3, -2)[..., :n, :]
    return codes.to(_FORMATS[fmt][1]), e.to(torch.int8)


def _values(codes, exps, block):
    e = exps.int().repeat_interleave(block, -1)[..., :codes.shape[-2], None]
    return codes.float() * _pow2(e)


def _requantised(x, fmt, block, dtype):
    """The values that rows x stand for once they are held in 8 bits."""
    n = x.shape[-2]
    y = _blocks(x.float(), block, n)
    e = _exponent(y.abs().amax((-1, -2)), fmt)[..., None, None]
    return (_code(y, e, fmt) * _pow2(e)).flatten(-3, -2)[..., :n, :].to(dtype)


def _plain_gather(st):
    c = st["c"]
    keep = c["keep"]
    n = st["n_keep"].transpose(0, 1)                                         # [L, batch(, heads)]
    n = (n if c["per_head"] else n[..., None].expand(-1, -1, c["kv_heads"])).flatten(0, 1)
    live = (torch.arange(keep, device=n.device) < n[..., None])[..., None]
    at = st["idx"][..., :keep, None].long().expand(-1, -1, -1, -1, c["head_dim"]) if c["idx"] else None
    pick = lambda x: (torch.gather(x, 3, at) if c["idx"] else x[..., :keep, :]).flatten(0, 1).float() * live  # noqa: E731
    return [_requantised(pick(st["k"]), c["fmt"], c["block"], _dtype(c)),
            _requantised(pick(st["v"]), c["fmt"], c["block"], _dtype(c)), n.contiguous()]


def _grown(codes, exps, new, lengths, c):
    """The blocks from the open one on, after `new` rows: their values, and rows behind the last one zero."""
    block, rows = c["block"], c["rows"]
    start = lengths // block * block
    n = rows + block
    row = start[..., None].long() + torch.arange(n, device=new.device)       # positions in the cache
    old = row < lengths[..., None]
    put = (row >= lengths[..., None]) & (row < lengths[..., None] + rows)
    inside = row.clamp(max=codes.shape[-2] - 1)
    # (the blocks as the cache counts them: n is not a multiple of a block, so the last one is filled up)
    held = torch.gather(codes.float(), 2, inside[..., None].expand(-1, -1, -1, codes.shape[-1])) * old[..., None]
    e_old = torch.gather(exps.int(), 2, (inside // block).clamp(max=exps.shape[-1] - 1))
    fresh = torch.gather(new.float(), 2, (row - lengths[..., None]).clamp(0, rows - 1)[..., None].expand(-1, -1, -1, new.shape[-1]))
    fresh = fresh * put[..., None]
    need = _exponent(_blocks(fresh, block, n).abs().amax((-1, -2)), c["fmt"])
    has_old = _blocks(old[..., None], block, n).any(-1).any(-1)
    first = _blocks(e_old[..., None], block, n)[..., 0, 0]
    e = torch.where(has_old, torch.maximum(need, first), need).repeat_interleave(block, -1)[..., :n]
    code = torch.where(old[..., None], _code(held, (e - e_old)[..., None], c["fmt"]), _code(fresh, e[..., None], c["fmt"]))
    return (code * _pow2(e[..., None])).to(_dtype(c))


def _plain_append(st):
    c, cache = st["c"], st["cache"]
    return [_grown(cache["k"], cache["k_exp"], st["k_new"], cache["lengths"], c),
            _grown(cache["v"], cache["v_exp"], st["v_new"], cache["lengths"], c), cache["lengths"] + c["rows"]]


def _plain_attend(st):
    c, cache = st["c"], st["cache"]
    b, h, rows, d = c["batch"], c["kv_heads"], c["rows"], c["head_dim"]
    group = c["q_heads"] // h
    k, v = _values(cache["k"], cache["k_exp"], c["block"]), _values(cache["v"], cache["v_exp"], c["block"])
    q = st["q"].float().reshape(b, h, group * rows, d)
    n = k.shape[-2]
    seen = cache["lengths"][..., None].long().expand(-1, -1, rows)
    if c["causal"]:
        seen = seen - (rows - 1) + torch.arange(rows, device=q.device)
    live = torch.arange(n, device=q.device) < seen.repeat(1, 1, group)[..., None]       # [b, h, group rows, n]
    s = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    s = s.masked_fill(~live, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top.masked_fill(top == -math.inf, 0.0))
    total = p.sum(-1, keepdim=True)
    p = p / total.masked_fill(total == 0, 1.0)
    v = v.masked_fill(~live.any(-2)[..., None], 0.0)
    out = torch.matmul(p, v).reshape(b, c["q_heads"], rows, d).to(_dtype(c))
    lse = (top + torch.log(total)).reshape(b, c["q_heads"], rows)
    if not c["weights"]:
        return [out, lse]
    # rows behind a head's last token are not written
    cached = torch.arange(n, device=q.device) < cache["lengths"][..., None]
    return [out, lse, (st["weight"] + p.sum(-2)) * cached]


def _plain_evict(st):
    c, cache = st["c"], st["cache"]
    n = torch.arange(st["weight"].shape[-1], device=st["weight"].device)
    lengths = cache["lengths"][..., None]
    w = st["weight"].masked_fill(n >= lengths - c["recent"], math.inf).masked_fill(n >= lengths, -math.inf)
    kept = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :c["budget"]]
    count = lengths.clamp(max=c["budget"])
    live = n[:c["budget"]] < count
    kept = kept.masked_fill(~live, w.shape[-1]).sort(-1).values
    at = kept.masked_fill(~live, 0)
    move = lambda x, e: torch.gather(_values(x, e, c["block"]), 2, at[..., None].expand(-1, -1, -1, c["head_dim"])) * live[..., None]  # noqa: E731
    weight = torch.gather(st["weight"], 2, at) * live
    return [_requantised(move(cache["k"], cache["k_exp"]), c["fmt"], c["block"], _dtype(c)),
            _requantised(move(cache["v"], cache["v_exp"]), c["fmt"], c["block"], _dtype(c)),
            kept.masked_fill(~live, -1).to(torch.int32), count[..., 0], weight]


# ---- the framework's operators --------------------------------------------------------------------------------------

def _cache(t, block):
    import paper_2509_05165_b200 as kvc
    return kvc.Cache(t["k"], t["v"], t["k_exp"], t["v_exp"], t["lengths"], block)


def _kept(st, name, make):
    """What a program makes once, before its first call, and keeps."""
    if name not in st:
        st[name] = make()
    return st[name]


def _own_rotary(st):
    import paper_2509_05165_b200 as kvc
    c = st["c"]
    lo, hi = _TURNS.get(c["scaling"], (0.0, 0.0))
    rope = _kept(st, "rope", lambda: kvc.Rotary(
        c["rot_dim"], theta=_THETA, interleaved=c["layout"] == "interleaved", scaling=c["scaling"], factor=_FACTOR,
        turns_low=lo, turns_high=hi, original_ctx=_ORIGINAL))
    kvc.kvc_rotary(rope, st["q"], st["k"], st["positions"], st["q_out"], st["k_out"])
    return [st["q_out"], st["k_out"]]


def _gather_plan(st):
    """The descriptor of the prefilled cache, a cache per layer, and all of them as one."""
    import paper_2509_05165_b200 as kvc
    c, t = st["c"], st["cache"]
    desc = kvc.kvc_desc_init(c["layers"], c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["n_ctx"], 1,
                             kvc.F32 if c["dtype"] == "f32" else kvc.BF16)
    part = lambda i: _cache({n: x[i * c["batch"]:(i + 1) * c["batch"]] for n, x in t.items()}, c["block"])  # noqa: E731
    return desc, [part(i) for i in range(c["layers"])], _cache(t, c["block"]), list(st["k"]), list(st["v"])


def _own_gather(st):
    import paper_2509_05165_b200 as kvc
    desc, caches, every, k, v = _kept(st, "plan", lambda: _gather_plan(st))
    kvc.kvc_cache_gather(desc, k, v, st["idx"], st["n_keep"], caches, per_head=st["c"]["per_head"])
    kvc.kvc_cache_read(every, st["k_out"], st["v_out"])
    return [st["k_out"], st["v_out"], st["cache"]["lengths"]]


def _own_append(st):
    import paper_2509_05165_b200 as kvc
    t, block = st["cache"], st["c"]["block"]
    before = _kept(st, "before", lambda: _cache(t, block))
    after = _kept(st, "after", lambda: _cache(dict(t, lengths=st["lengths_out"]), block))
    kvc.kvc_cache_append(before, st["k_new"], st["v_new"], lengths_out=st["lengths_out"])
    kvc.kvc_cache_read(after, st["k_out"], st["v_out"], first=st["first"])
    return [st["k_out"], st["v_out"], st["lengths_out"]]


def _own_attend(st):
    import paper_2509_05165_b200 as kvc
    c = st["c"]
    cache = _kept(st, "handle", lambda: _cache(st["cache"], c["block"]))
    ws = _kept(st, "ws", lambda: torch.empty(kvc.kvc_attend_workspace_size(cache, st["q"], c["weights"]), dtype=torch.uint8,
                                             device=st["q"].device))
    kvc.kvc_attend(cache, st["q"], st["out"], lse=st["lse"], weight=st.get("weight"), weight_out=st.get("weight_out"),
                   causal=c["causal"], workspace=ws)
    return [st["out"], st["lse"]] + ([st["weight_out"]] if c["weights"] else [])


def _own_evict(st):
    import paper_2509_05165_b200 as kvc
    c = st["c"]
    src = _kept(st, "src", lambda: _cache(st["cache"], c["block"]))
    dst = _kept(st, "to", lambda: _cache(st["dst"], c["block"]))
    kvc.kvc_evict(src, dst, st["weight"], c["budget"], c["recent"], st["idx"], weight_out=st["weight_out"])
    kvc.kvc_cache_read(dst, st["k_out"], st["v_out"])
    return [st["k_out"], st["v_out"], st["idx"], st["dst"]["lengths"], st["weight_out"]]


_PLAIN = dict(rotary=_plain_rotary, gather=_plain_gather, append=_plain_append, attend=_plain_attend, evict=_plain_evict)
_OWN = dict(rotary=_own_rotary, gather=_own_gather, append=_own_append, attend=_own_attend, evict=_own_evict)


def run(state):
    if own:
        return _OWN[state["c"]["kind"]](state)
    return _PLAIN[state["c"]["kind"]](state)


# ---- work -----------------------------------------------------------------------------------------------------------

def work(case):
    c = dict(_BASE, **case)
    e = 4.0 if c["dtype"] == "f32" else 2.0
    units, d = c["batch"] * c["kv_heads"], c["head_dim"]
    if c["kind"] == "rotary":
        values = float(c["batch"] * (c["q_heads"] + c["kv_heads"]) * c["rows"] * d)
        return {"bytes": 2.0 * e * values, "flops": 3.0 * values * c["rot_dim"] / d}
    if c["kind"] == "gather":       # half of the places are kept on average; every place's values are written
        values = 2.0 * c["layers"] * units * c["keep"] * d
        return {"bytes": values * (0.5 * e + 0.5 + e), "flops": values}
    if c["kind"] == "append":       # the new rows, the codes of the open block and theirs, the values of both
        values = 2.0 * units * c["rows"] * d
        return {"bytes": values * (e + 1.0 + e) + 2.0 * units * c["block"] * d * (0.5 + e), "flops": values}
    tokens = float(c["length"] * units)
    if c["ragged"]:                 # the mean of a length that is spread over its logarithm, and one full sequence
        mean = (c["length"] - 1.0) / math.log(c["length"] + 1.0) if c["length"] > 1 else 1.0
        tokens = c["kv_heads"] * (c["length"] + max(0, c["batch"] - 2) * mean)
    if c["kind"] == "attend":
        rows = c["rows"] * c["q_heads"] // c["kv_heads"]
        return {"bytes": 2.0 * tokens * d + (8.0 * tokens if c["weights"] else 0.0) + 2.0 * e * units * rows * d,
                "flops": 4.0 * tokens * rows * d}
    kept = min(tokens, float(units * c["budget"]))
    return {"bytes": 4.0 * tokens + 2.0 * kept * d * (1.0 + 1.0) + 2.0 * units * c["budget"] * d * e + 12.0 * kept, "flops": tokens}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    def two(e):
        return ((e.long() + 1023) << 52).view(torch.float64)          # 2^e, exactly

    def held(x, fmt):
        """Rows of one block [..., block, d] in 64 bits -> what they stand for once held in 8 bits, and the exponent."""
        qmax = _FORMATS[fmt][0]
        amax = x.abs().amax((-1, -2), keepdim=True)
        e = torch.ceil(torch.log2(amax.clamp(min=1e-300) / qmax)).clamp(_E_MIN, _E_MAX)
        e = torch.where(amax > qmax * two(e), e + 1, e)          # (the logarithm next to a power of two)
        e = torch.where((amax <= qmax * two(e - 1)) & (e > _E_MIN), e - 1, e)
        return nearest(x, e, fmt), e

    def nearest(x, e, fmt):
        y = x * two(-e)
        if fmt == "int8":
            return torch.round(y) * two(e)
        step = two(torch.frexp(y.abs().clamp(min=0.015625)).exponent - 4)       # (an eighth of the power of two below)
        return torch.round(y / step) * step * two(e)

    def rotary(c, st):
        i = torch.arange(0, c["rot_dim"], 2, device="cuda").double()
        f = torch.exp(-i / c["rot_dim"] * math.log(_THETA))
        factor = 1.0
        if c["scaling"] == "linear":
            f = f / _FACTOR
        elif c["scaling"] == "banded":
            lo, hi = _TURNS["banded"]
            wave = 2.0 * math.pi / f
            smooth = (_ORIGINAL / wave - lo) / (hi - lo)
            f = torch.where(wave < _ORIGINAL / hi, f, torch.where(wave > _ORIGINAL / lo, f / _FACTOR, (1 - smooth) * f / _FACTOR + smooth * f))
        elif c["scaling"] == "yarn":
            lo, hi = _TURNS["yarn"]
            pair = lambda turns: c["rot_dim"] / 2.0 * math.log(_ORIGINAL / (2.0 * math.pi * turns)) / math.log(_THETA)  # noqa: E731
            a, b = max(math.floor(pair(hi)), 0), min(math.ceil(pair(lo)), c["rot_dim"] - 1)
            share = torch.clamp((i / 2 - a) / max(b - a, 0.001), 0, 1)
            f, factor = f / _FACTOR * share + f * (1 - share), 1.0 + 0.1 * math.log(_FACTOR)
        turn = torch.polar(torch.full((), factor, device="cuda").double().expand(st["positions"].shape + f.shape),
                           st["positions"].double()[..., None] * f)[:, None]
        out = []
        for x in (st["q"].double(), st["k"].double()):
            z = x[..., :c["rot_dim"]]
            z = torch.stack(z.chunk(2, -1), -1) if c["layout"] == "half" else z.unflatten(-1, (-1, 2))
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
            z = torch.cat([z[..., 0], z[..., 1]], -1) if c["layout"] == "half" else z.flatten(-2)
            out.append(torch.cat([z, x[..., c["rot_dim"]:]], -1))
        return out

    def gather(c, st):
        n = st["n_keep"].cpu()
        outs = [torch.zeros_like(st["k_out"], dtype=torch.float64) for _ in range(2)]
        for layer in range(c["layers"]):
            for b in range(c["batch"]):
                for h in range(c["kv_heads"]):
                    m = int(n[b, layer, h] if c["per_head"] else n[b, layer])
                    at = st["idx"][layer, b, h, :m].long() if c["idx"] else slice(0, m)
                    for out, src in zip(outs, (st["k"], st["v"])):
                        rows = src[layer, b, h][at].double()
                        full = torch.zeros((-(-m // c["block"]) * c["block"], c["head_dim"]), dtype=torch.float64, device="cuda")
                        full[:m] = rows
                        out[layer * c["batch"] + b, h, :m] = held(full.view(-1, c["block"], c["head_dim"]), c["fmt"])[0].flatten(0, 1)[:m]
        return outs + [None]

    def append(c, st):
        t, block, outs = st["cache"], c["block"], []
        for codes, exps, new in ((t["k"], t["k_exp"], st["k_new"]), (t["v"], t["v_exp"], st["v_new"])):
            out = torch.zeros(st["k_out"].shape, dtype=torch.float64, device="cuda")
            for b in range(c["batch"]):
                n = int(t["lengths"][b, 0])             # (a sequence's heads are equally long here)
                have, start = n % block, n // block * block
                was = exps[b, :, n // block].double()[:, None, None] if have else None
                x = new[b].double()
                if have:
                    rest = x[:, :block - have]
                    e = torch.maximum(held(rest, c["fmt"])[1], was)
                    out[b, :, :have] = nearest(codes[b, :, start:n].double() * two(was), e, c["fmt"])
                    out[b, :, have:have + rest.shape[1]] = nearest(rest, e, c["fmt"])
                    x = x[:, block - have:]
                at = block if have else 0
                for r0 in range(0, x.shape[1], block):
                    piece = x[:, r0:r0 + block]
                    out[b, :, at + r0:at + r0 + piece.shape[1]] = held(piece, c["fmt"])[0]
            outs.append(out)
        return outs + [None]

    def attend(c, st):
        t, h, rows = st["cache"], c["kv_heads"], c["rows"]
        group = c["q_heads"] // h
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(st["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
        weight = torch.zeros(st["weight"].shape, dtype=torch.float64, device="cuda") if c["weights"] else None
        for b in range(c["batch"]):
            n = int(t["lengths"][b, 0])
            if n == 0:
                continue
            block = torch.arange(n, device="cuda") // c["block"]
            k = t["k"][b, :, :n].double() * two(t["k_exp"][b])[:, block, None]
            v = t["v"][b, :, :n].double() * two(t["v_exp"][b])[:, block, None]
            if weight is not None:
                weight[b, :, :n] = st["weight"][b, :, :n].double()
            for r in range(rows):
                m = n - (rows - 1 - r) if c["causal"] else n
                if m <= 0:
                    continue
                q = st["q"][b, :, r].double().reshape(h, group, -1)
                s = torch.einsum("hgd,hnd->hgn", q, k[:, :m]) / math.sqrt(c["head_dim"])
                p = torch.softmax(s, -1)
                out[b, :, r] = torch.einsum("hgn,hnd->hgd", p, v[:, :m]).flatten(0, 1)
                lse[b, :, r] = torch.logsumexp(s, -1).flatten()
                if weight is not None:
                    weight[b, :, :m] += p.sum(1)
        return [out, lse] + ([weight] if c["weights"] else [])

    def evict(c, st):
        t = st["cache"]
        outs = [torch.zeros(st["k_out"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
        weight = torch.zeros(st["weight_out"].shape, dtype=torch.float64, device="cuda")
        for b in range(c["batch"]):
            n = int(t["lengths"][b, 0])
            m = min(n, c["budget"])
            if m == 0:
                continue
            for h in range(c["kv_heads"]):
                w = st["weight"][b, h, :n].double()
                free = max(0, n - c["recent"]) if n > c["budget"] else 0
                heavy = torch.argsort(-w[:free], stable=True)[:m - (n - free)]
                at = torch.cat([heavy.sort().values, torch.arange(free, n, device="cuda")])
                weight[b, h, :m] = w[at]
                for out, codes, exps in ((outs[0], t["k"], t["k_exp"]), (outs[1], t["v"], t["v_exp"])):
                    x = codes[b, h, at].double() * two(exps[b, h, at // c["block"]])[:, None]
                    full = torch.zeros((-(-m // c["block"]) * c["block"], c["head_dim"]), dtype=torch.float64, device="cuda")
                    full[:m] = x
                    out[b, h, :m] = held(full.view(-1, c["block"], c["head_dim"]), c["fmt"])[0].flatten(0, 1)[:m]
        return outs + [None, None, weight]

    st = prepare(case, seed)
    c = st["c"]
    return dict(rotary=rotary, gather=gather, append=append, attend=attend, evict=evict)[c["kind"]](c, st)
