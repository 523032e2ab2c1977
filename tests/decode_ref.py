"""Plain definitions of the decoding operators in 64 bits (CPU tensors), written apart from the kernels, and their inputs."""
import math

import torch

QMAX = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}
E_MIN, E_MAX = -100, 121


def frequencies(rope):
    """Angle per position of every pair, and the factor on the rotated values."""
    i = torch.arange(rope.rot_dim // 2, dtype=torch.float64)
    f = torch.tensor([rope.theta ** (-2.0 * int(j) / rope.rot_dim) for j in i], dtype=torch.float64)
    m = 1.0
    if rope.scaling == "linear":
        f = f / rope.factor
    elif rope.scaling == "banded":
        turns = rope.original_ctx * f / (2 * math.pi)
        share = ((turns - rope.turns_low) / (rope.turns_high - rope.turns_low)).clamp(0, 1)
        f = share * f + (1 - share) * f / rope.factor
    elif rope.scaling == "yarn":
        pair = lambda t: rope.rot_dim * math.log(rope.original_ctx / (2 * math.pi * t)) / (2 * math.log(rope.theta))  # noqa: E731
        lo, hi = max(math.floor(pair(rope.turns_high)), 0), min(math.ceil(pair(rope.turns_low)), rope.rot_dim - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f, m = f * (1 - ramp) + f / rope.factor * ramp, 0.1 * math.log(rope.factor) + 1
    return f, (rope.mscale or m)


def rotate(x, positions, rope, inverse=False):
    """x [batch, heads, rows, d] in 64 bits; positions [batch, rows]."""
    f, m = frequencies(rope)
    t = positions.double()[:, None, :, None] * f * (-1.0 if inverse else 1.0)
    c, s = torch.cos(t) * m, torch.sin(t) * m
    x = x.double()
    y, r = x.clone(), rope.rot_dim
    one, two = (slice(0, r, 2), slice(1, r, 2)) if rope.interleaved else (slice(0, r // 2), slice(r // 2, r))
    y[..., one] = x[..., one] * c - x[..., two] * s
    y[..., two] = x[..., two] * c + x[..., one] * s
    return y


def exponent(amax, dtype):
    """Smallest e in [E_MIN, E_MAX] with amax <= qmax 2^e, by trying (amax: a Python float)."""
    if amax == 0.0:
        return E_MIN
    e = max(E_MIN, min(E_MAX, math.frexp(amax)[1] - math.frexp(QMAX[dtype])[1] - 1))
    while e < E_MAX and amax > math.ldexp(QMAX[dtype], e):
        e += 1
    return e


def round_code(y, dtype):
    """Codes (as 64-bit numbers) of y: nearest, ties to even, held at the largest."""
    y = y.clamp(-QMAX[dtype], QMAX[dtype])
    if dtype == torch.int8:
        return torch.round(y)
    step = torch.ldexp(torch.ones_like(y), (torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4))
    return torch.round(y / step) * step


def hold(x, dtype):
    """Rows of one block -> (codes, e)."""
    e = exponent(float(x.abs().max()) if x.numel() else 0.0, dtype)
    return round_code(x.double() * 2.0 ** -e, dtype), e


class Held:
    """One head's K or V rows as an 8-bit cache holds them."""

    def __init__(self, dtype, block):
        self.dtype, self.block, self.codes, self.exps = dtype, block, [], []

    def fill(self, x):
        self.codes, self.exps = [], []
        for r in range(0, x.shape[0], self.block):
            c, e = hold(x[r:r + self.block], self.dtype)
            self.codes.append(c)
            self.exps.append(e)
        return self

    def append(self, x):
        while x.shape[0]:
            room = self.block - self.codes[-1].shape[0] if self.codes else 0
            if room:
                part, x = x[:room].double(), x[room:]
                was = self.exps[-1]
                e = max(was, exponent(float(part.abs().max()), self.dtype))
                old = self.codes[-1] if e == was else round_code(self.codes[-1] * 2.0 ** max(was - e, -126), self.dtype)
                self.codes[-1], self.exps[-1] = torch.cat([old, round_code(part * 2.0 ** -e, self.dtype)]), e
            else:
                c, e = hold(x[:self.block], self.dtype)
                self.codes.append(c)
                self.exps.append(e)
                x = x[self.block:]
        return self

    def values(self, d=0):
        return torch.cat([c * 2.0 ** e for c, e in zip(self.codes, self.exps)]) if self.codes else torch.zeros((0, d), dtype=torch.float64)


def cache_values(cache):
    """Values [batch, heads, capacity, d] of a kvc.Cache's codes in 64 bits (rows behind a length: whatever is there)."""
    out = []
    for codes, exps in ((cache.k, cache.k_exp), (cache.v, cache.v_exp)):
        e = exps.cpu().long().repeat_interleave(cache.block, -1)[..., :codes.shape[2], None]
        out.append(codes.cpu().to(torch.float64) * torch.pow(torch.tensor(2.0, dtype=torch.float64), e.double()))
    return out


def attend(q, k, v, lengths, causal, scale, counts=None, step=None, small=0.0):
    """q [b, hq, rows, d], k, v [b, h, n, d], all in 64 bits.  Returns out, lse, the weight each token gets, sum p |v| (what
    errors of p are measured against) and the largest sum |q k| scale (what errors of a logit are).  step [b, h, n]: what one
    unit of a V code stands for; sum p |v| then gets a term for P's smallest steps, `small` of the row's largest p times step
    for each token and codes of up to 448."""
    b, hq, rows, d = q.shape
    h, n = k.shape[1], k.shape[2]
    out, lse = torch.zeros_like(q), torch.full((b, hq, rows), -math.inf, dtype=torch.float64)
    weight, mass, size = torch.zeros((b, h, n), dtype=torch.float64), torch.zeros_like(q), 0.0
    for i in range(b):
        nr = rows if counts is None else int(counts[i])
        for j in range(hq):
            g = j // (hq // h)
            m = int(lengths[i, g])
            for r in range(nr):
                seen = m - (nr - 1 - r) if causal else m
                if seen <= 0:
                    continue
                kk, vv = k[i, g, :seen], v[i, g, :seen]
                s = kk @ q[i, j, r] * scale
                size = max(size, float((kk.abs() @ q[i, j, r].abs()).max() * scale))
                p = torch.softmax(s, 0)
                out[i, j, r], mass[i, j, r] = p @ vv, p @ vv.abs()
                if step is not None:
                    mass[i, j, r] += seen * small * 448.0 * float((p * step[i, g, :seen]).max())
                lse[i, j, r] = torch.logsumexp(s, 0)
                weight[i, g, :seen] += p
    return out, lse, weight, mass, size


def evict(weight, n, budget, recent):
    """Kept positions of one head, ascending."""
    if n <= budget:
        return list(range(n))
    free = n - recent
    heavy = sorted(range(free), key=lambda i: (-float(weight[i]), i))[:budget - recent]
    return sorted(heavy) + list(range(free, n))


def spread_rows(gen, *shape):
    """Normal rows of very different sizes."""
    return torch.randn(shape, generator=gen) * torch.exp(2.0 * torch.randn(shape[:-1] + (1,), generator=gen))
