"""Decoding from a compressed cache: the binding of kvc.h's 8-bit cache, its attention and eviction, and rotary positions.

Same names as the C entry points; tensors are checked for type, shape, layout and device here, values and sizes in the
library.  A decoding step makes several calls per layer whose kernels take microseconds, so what a combination of types,
shapes, strides and devices was checked for and turned into is kept (by these and the options' values, never by a tensor's
identity or address) with the object that the calls share, and looked up by the next call.  Everything runs on ``stream``
(default: the current one), which has to be a stream of the tensors' device, and that device the current one.

    cache = kvc.alloc_cache(batch, n_kv_heads, head_dim, capacity, device=dev)      # one layer
    kvc.kvc_cache_gather(desc, k, v, idx, n_keep, caches)                            # kept rows, all layers
    kvc.kvc_rotary(rope, q, k_new, positions, q, k_new)                              # one step of one layer
    kvc.kvc_cache_append(cache, k_new, v_new, weight=weight)
    kvc.kvc_attend(cache, q, out, weight=weight, workspace=ws)
    kvc.kvc_evict(cache, spare, weight, budget, recent, idx, weight_out=spare_weight)    # now and then
"""
from __future__ import annotations

import ctypes as C
import dataclasses
from typing import Optional, Sequence

import torch

from .binding import BF16, F32, KvcAttendDesc, KvcCache, KvcError, KvcRope, KvcRopeDesc, _check, _load, _ptr_array, _stream

INT8, E4M3 = 0, 1
_SCALING = {"none": 0, "linear": 1, "banded": 2, "yarn": 3}
_FORMATS = {torch.int8: INT8, torch.float8_e4m3fn: E4M3}
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


def _refuse(cond: bool, message: str, *args) -> None:
    if cond:
        raise KvcError(-1, message % args if args else message)


def _dtype(t: torch.Tensor, name: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise KvcError(-1, "%s must be bf16 or fp32, not %s" % (name, t.dtype))
    return code


def _rows4(t: torch.Tensor, name: str, batch: int, heads: Optional[int], rows: Optional[int], d: int, dtype=None) -> None:
    """[batch, heads, rows, d] with contiguous rows."""
    ok = (t.dim() == 4 and t.shape[0] == batch and t.shape[3] == d and (heads is None or t.shape[1] == heads)
          and (rows is None or t.shape[2] == rows))
    _refuse(not ok, "%s has shape %s, not [%s, %s, %s, %s]", name, tuple(t.shape), batch, heads or "heads", rows or "rows", d)
    _refuse(t.stride(3) != 1, "%s: a row's entries must be contiguous", name)
    _refuse(dtype is not None and t.dtype != dtype, "%s must be %s, not %s", name, dtype, t.dtype)


def _dense(t: Optional[torch.Tensor], name: str, dtype, *shape) -> None:
    if t is None:
        return
    _refuse(t.dtype != dtype, "%s must be %s, not %s", name, dtype, t.dtype)
    _refuse(tuple(t.shape) != shape, "%s has shape %s, not %s", name, tuple(t.shape), shape)
    _refuse(not t.is_contiguous(), "%s must be contiguous", name)


def _sig(t: Optional[torch.Tensor]):
    """All that the checks go by."""
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device())


class _Plans(dict):
    """What calls with the same signature share; forgotten when there are very many of them."""

    def keep(self, key, plan):
        if len(self) >= 512:
            self.clear()
        self[key] = plan
        return plan


def _one_device(first: torch.Tensor, *others: Optional[torch.Tensor]) -> int:
    dev = first.get_device()
    for t in others:
        if t is not None and t.get_device() != dev:
            raise KvcError(-1, "tensors on different devices: %s and %s" % (first.device, t.device))
    return dev


_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _launch_stream(dev: int, stream):
    """The stream to launch on; the tensors' device has to be the current one (launches go there)."""
    if dev < 0:
        # (host memory: without a GPU the library says what else is wrong, and that there is none; with one it must not see it)
        _refuse(torch.cuda.is_available(), "tensors in host memory")
        return _stream(stream)
    if dev != _get_device():
        raise KvcError(-1, "tensors on cuda:%d, which is not the current device" % dev)
    if stream is None and _raw_stream is not None:
        return _raw_stream(dev)
    return _stream(stream)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _strides(t: torch.Tensor):
    # (a dimension of one row may have any stride; slot 0 at 0 would mean dense, so a stride for a batch of one is made up)
    d = t.shape[3]
    s = [t.stride(i) if t.shape[i] > 1 else 0 for i in range(3)]
    if s[2] == 0 and t.shape[2] == 1:
        s[2] = d
    if s[0] == 0:
        _refuse(t.shape[0] > 1, "a batch of one row repeated (stride 0) is not supported")
        s[0] = max(s[1] * t.shape[1], s[2] * t.shape[2])
    return (C.c_int64 * 3)(*s)


class Cache:
    """An 8-bit cache of one layer (or of layers laid out as one batch) over tensors that the caller keeps.

    k, v      [batch, n_kv_heads, capacity, head_dim], ``torch.int8`` or ``torch.float8_e4m3fn``; a token's entries contiguous
    k_exp, v_exp   [batch, n_kv_heads, ceil(capacity / block)] int8; lengths [batch, n_kv_heads] int32; contiguous
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor, v_exp: torch.Tensor, lengths: torch.Tensor, block: int):
        _refuse(k.dim() != 4, "k has %d dimensions, not 4", k.dim())
        fmt = _FORMATS.get(k.dtype)
        _refuse(fmt is None, "k must be int8 or float8_e4m3fn, not %s", k.dtype)
        _refuse(block not in (16, 32, 64, 128), "block must be 16, 32, 64 or 128")
        b, h, cap, d = k.shape
        _rows4(k, "k", b, h, cap, d)
        _rows4(v, "v", b, h, cap, d, k.dtype)
        blocks = -(-cap // block)
        _dense(k_exp, "k_exp", torch.int8, b, h, blocks)
        _dense(v_exp, "v_exp", torch.int8, b, h, blocks)
        _dense(lengths, "lengths", torch.int32, b, h)
        dev = k.get_device()
        for t in (v, k_exp, v_exp, lengths):
            _refuse(t.get_device() != dev, "the cache's tensors are on different devices")
        ks = _strides(k)
        _refuse(list(ks) != list(_strides(v)), "k and v have different strides")
        self.k, self.v, self.k_exp, self.v_exp, self.lengths, self.block = k, v, k_exp, v_exp, lengths, block
        self.batch, self.n_kv_heads, self.capacity, self.head_dim, self.format = b, h, cap, d, fmt
        self.struct = KvcCache(b, h, d, block, fmt, 0, cap, ks, k.data_ptr(), v.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(),
                               lengths.data_ptr())
        self.ref, self.plans, self.device = C.byref(self.struct), _Plans(), dev

    @property
    def bytes(self) -> int:
        return 2 * (self.k.numel() + self.k_exp.numel())


def alloc_cache(batch: int, n_kv_heads: int, head_dim: int, capacity: int, block: int = 64, dtype=torch.float8_e4m3fn, device="cuda") -> Cache:
    """An empty cache."""
    codes = lambda: torch.zeros((batch, n_kv_heads, capacity, head_dim), dtype=dtype, device=device)  # noqa: E731
    exps = lambda: torch.zeros((batch, n_kv_heads, -(-capacity // block)), dtype=torch.int8, device=device)  # noqa: E731
    return Cache(codes(), codes(), exps(), exps(), torch.zeros((batch, n_kv_heads), dtype=torch.int32, device=device), block)


@dataclasses.dataclass(frozen=True)
class Rotary:
    """Rotary positions of ``rot_dim`` of a head's entries; see ``kvc_rope_scaling`` for the scalings."""
    rot_dim: int
    theta: float = 10000.0
    interleaved: bool = False
    scaling: str = "none"            # "none" | "linear" | "banded" | "yarn"
    factor: float = 1.0
    turns_low: float = 1.0
    turns_high: float = 4.0
    original_ctx: float = 8192.0
    mscale: float = 0.0              # 0: the scaling's own

    def __post_init__(self):
        _refuse(self.scaling not in _SCALING, "unknown scaling %r", self.scaling)
        rope = KvcRope()
        _check(_load().kvc_rope_init(C.byref(rope), self.rot_dim, int(self.interleaved), self.theta, _SCALING[self.scaling], self.factor,
                                     self.turns_low, self.turns_high, self.original_ctx, self.mscale))
        object.__setattr__(self, "struct", rope)
        object.__setattr__(self, "ref", C.byref(rope))
        object.__setattr__(self, "plans", _Plans())

    def __reduce__(self):                # (copies and pickles are made from the fields: the rest holds addresses)
        return Rotary, tuple(getattr(self, f.name) for f in dataclasses.fields(self))


def _rotary_plan(q, k, positions, q_out, k_out, inverse):
    x = q if q is not None else k
    _refuse(x is None, "q and k are both None")
    _refuse(x.dim() != 4, "q and k have four dimensions")
    b, _, rows, d = x.shape
    code = _dtype(x, "q or k")
    _refuse(q is None and q_out is not None or k is None and k_out is not None, "an output without its input")
    for t, o, name in ((q, q_out, "q"), (k, k_out, "k")):
        if t is not None:
            _rows4(t, name, b, None, rows, d, x.dtype)
            _rows4(o, name + "_out", b, t.shape[1], rows, d, x.dtype)
    _refuse(positions.dtype != torch.int64, "positions must be int64, not %s", positions.dtype)
    _refuse(tuple(positions.shape) not in ((rows,), (b, rows), (1, rows)), "positions has shape %s, not [%d] or [%d, %d]",
            tuple(positions.shape), rows, b, rows)
    _refuse(rows > 1 and positions.stride(-1) != 1, "a sequence's positions must be contiguous")
    desc = KvcRopeDesc(b, q.shape[1] if q is not None else 0, k.shape[1] if k is not None else 0, d, rows, code, int(inverse), 0)
    if q is not None:
        desc.q_stride, desc.q_out_stride = _strides(q), _strides(q_out)
    if k is not None:
        desc.k_stride, desc.k_out_stride = _strides(k), _strides(k_out)
    per_sequence = positions.stride(0) if positions.dim() == 2 and positions.shape[0] > 1 else 0
    return C.byref(desc), per_sequence, _one_device(x, k, positions, q_out, k_out)


def kvc_rotary(rope: Rotary, q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: torch.Tensor,
               q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, inverse: bool = False, stream=None) -> None:
    """Turn q [batch, n_q_heads, rows, head_dim] and k [batch, n_kv_heads, rows, head_dim] (either may be None) by
    ``positions`` ([rows] or [batch, rows], int64).  Outputs default to their inputs (in place)."""
    if q_out is None:
        q_out = q
    if k_out is None:
        k_out = k
    inverse = bool(inverse)
    key = (_sig(q), _sig(k), _sig(positions), _sig(q_out), _sig(k_out), inverse)
    plan = rope.plans.get(key) or rope.plans.keep(key, _rotary_plan(q, k, positions, q_out, k_out, inverse))
    _check(_load().kvc_rotary(rope.ref, plan[0], _ptr(q), _ptr(k), positions.data_ptr(), plan[1], _ptr(q_out), _ptr(k_out),
                              _launch_stream(plan[2], stream)))


_gather_plans = _Plans()


def _gather_plan(desc, k, v, idx, n_keep, caches, per_head, device_status):
    L, b, h, n, d = desc.n_layers, desc.batch, desc.n_kv_heads, desc.n_ctx, desc.head_dim
    _refuse(not (len(k) == len(v) == len(caches) == L), "k, v and caches hold one entry per layer (%d)", L)
    dtype = torch.float32 if desc.dtype == F32 else torch.bfloat16
    given = tuple(desc.kv_stride) if desc.kv_stride[0] else (h * n * d, n * d, d)
    for t in (*k, *v):
        _rows4(t, "k or v", b, h, n, d, dtype)
        _refuse(any(t.shape[i] > 1 and t.stride(i) != given[i] for i in range(3)), "k or v has other strides than desc.kv_stride")
    _dense(idx, "idx", torch.int32, L, b, h, n)
    _dense(n_keep, "n_keep", torch.int32, *((b, L, h) if per_head else (b, L)))
    _refuse(device_status is not None and device_status.dtype != torch.int32, "device_status must be int32")
    return (_one_device(k[0], *k, *v, idx, n_keep, device_status, *(c.k for c in caches)),)


def kvc_cache_gather(desc, k: Sequence[torch.Tensor], v: Sequence[torch.Tensor], idx: Optional[torch.Tensor],
                     n_keep: Optional[torch.Tensor], caches: Sequence[Cache], per_head: bool = False,
                     device_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """``kvc_gather`` into 8-bit caches, one per layer.  idx [L, batch, Hkv, N] int32 or None; n_keep [batch, L] (or, with
    ``per_head``, [batch, L, Hkv]) int32 or None.  device_status: int32, becomes KVC_ERR_CAPACITY if rows did not fit, KVC_ERR_NOT_FINITE (over 0 only)
    if kept rows held infinities or NaN."""
    per_head = bool(per_head)
    key = (bytes(desc), per_head, tuple(map(_sig, k)), tuple(map(_sig, v)), _sig(idx), _sig(n_keep), _sig(device_status),
           tuple([c.device for c in caches]))
    plan = _gather_plans.get(key) or _gather_plans.keep(key, _gather_plan(desc, k, v, idx, n_keep, caches, per_head, device_status))
    structs = (KvcCache * len(caches))(*[c.struct for c in caches])
    _check(_load().kvc_cache_gather(C.byref(desc), _ptr_array(k), _ptr_array(v), _ptr(idx), _ptr(n_keep), int(per_head), structs,
                                    _ptr(device_status), _launch_stream(plan[0], stream)))


def _append_plan(cache, k_new, v_new, n_new, lengths_out, weight, device_status):
    b, h = cache.batch, cache.n_kv_heads
    code = _dtype(k_new, "k_new")
    _rows4(k_new, "k_new", b, h, None, cache.head_dim)
    _rows4(v_new, "v_new", b, h, k_new.shape[2], cache.head_dim, k_new.dtype)
    strides = _strides(k_new)
    _refuse(list(strides) != list(_strides(v_new)), "k_new and v_new have different strides")
    _dense(n_new, "n_new", torch.int32, b)
    _dense(lengths_out, "lengths_out", torch.int32, b, h)
    _dense(weight, "weight", torch.float32, b, h, cache.capacity)
    _refuse(device_status is not None and device_status.dtype != torch.int32, "device_status must be int32")
    return code, k_new.shape[2], strides, _one_device(cache.k, k_new, v_new, n_new, lengths_out, weight, device_status)


def kvc_cache_append(cache: Cache, k_new: torch.Tensor, v_new: torch.Tensor, n_new: Optional[torch.Tensor] = None,
                     lengths_out: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                     device_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Rows of new tokens [batch, Hkv, rows, head_dim] behind the ones in use; ``n_new`` [batch] int32 of them per sequence.
    device_status as in ``kvc_cache_gather``."""
    key = ("append", _sig(k_new), _sig(v_new), _sig(n_new), _sig(lengths_out), _sig(weight), _sig(device_status))
    plan = cache.plans.get(key) or cache.plans.keep(key, _append_plan(cache, k_new, v_new, n_new, lengths_out, weight, device_status))
    _check(_load().kvc_cache_append(cache.ref, k_new.data_ptr(), v_new.data_ptr(), plan[0], plan[1], plan[2], _ptr(n_new), _ptr(lengths_out),
                                    _ptr(weight), _ptr(device_status), _launch_stream(plan[3], stream)))


def _read_plan(cache, k_out, v_out, first):
    x = k_out if k_out is not None else v_out
    _refuse(x is None, "k_out and v_out are both None")
    code = _dtype(x, "k_out or v_out")
    _refuse(x.dim() != 4, "k_out and v_out have four dimensions")
    for t in (k_out, v_out):
        _dense(t, "k_out or v_out", x.dtype, cache.batch, cache.n_kv_heads, x.shape[2], cache.head_dim)
    _dense(first, "first", torch.int32, cache.batch, cache.n_kv_heads)
    return code, x.shape[2], _one_device(cache.k, k_out, v_out, first)


def kvc_cache_read(cache: Cache, k_out: Optional[torch.Tensor], v_out: Optional[torch.Tensor], first: Optional[torch.Tensor] = None,
                   stream=None) -> None:
    """Values of the rows first[b, h] .. into k_out, v_out [batch, Hkv, rows, head_dim] (bf16 or fp32, contiguous)."""
    key = ("read", _sig(k_out), _sig(v_out), _sig(first))
    plan = cache.plans.get(key) or cache.plans.keep(key, _read_plan(cache, k_out, v_out, first))
    _check(_load().kvc_cache_read(cache.ref, _ptr(first), plan[1], plan[0], _ptr(k_out), _ptr(v_out), _launch_stream(plan[2], stream)))


def _attend_desc(cache: Cache, q: torch.Tensor, out: Optional[torch.Tensor], causal: bool, scale: float) -> KvcAttendDesc:
    code = _dtype(q, "q")
    _rows4(q, "q", cache.batch, None, None, cache.head_dim)
    desc = KvcAttendDesc(q.shape[1], q.shape[2], code, int(causal), scale, 0, _strides(q))
    if out is not None:
        _rows4(out, "out", cache.batch, q.shape[1], q.shape[2], cache.head_dim, q.dtype)
        desc.out_stride = _strides(out)
    return desc


def kvc_attend_workspace_size(cache: Cache, q: torch.Tensor, with_weight: bool) -> int:
    """Bytes of scratch ``kvc_attend`` needs for queries of q's shape; with_weight: with the tokens' weights."""
    out = C.c_size_t(0)
    desc = _attend_desc(cache, q, None, True, 0.0)
    _check(_load().kvc_attend_workspace_size(cache.ref, C.byref(desc), int(with_weight), C.byref(out)))
    return int(out.value)


def _attend_plan(cache, q, out, lse, weight, weight_out, row_counts, causal, scale, workspace):
    b, h = cache.batch, cache.n_kv_heads
    desc = _attend_desc(cache, q, out, causal, scale)
    _dense(lse, "lse", torch.float32, b, q.shape[1], q.shape[2])
    _dense(weight, "weight", torch.float32, b, h, cache.capacity)
    _dense(weight_out, "weight_out", torch.float32, b, h, cache.capacity)
    _dense(row_counts, "row_counts", torch.int32, b)
    _refuse(workspace is not None and not workspace.is_contiguous(), "workspace must be contiguous")
    dev = _one_device(cache.k, q, out, lse, weight, weight_out, row_counts, workspace)
    return C.byref(desc), 0 if workspace is None else workspace.numel() * workspace.element_size(), dev


def kvc_attend(cache: Cache, q: torch.Tensor, out: torch.Tensor, lse: Optional[torch.Tensor] = None,
               weight: Optional[torch.Tensor] = None, weight_out: Optional[torch.Tensor] = None,
               row_counts: Optional[torch.Tensor] = None, causal: bool = True, scale: float = 0.0,
               workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Attention of q [batch, n_q_heads, rows, head_dim] over the cache into out.  lse [batch, n_q_heads, rows] fp32.
    weight [batch, Hkv, capacity] fp32: the tokens' running weight, added to in place, or into ``weight_out``."""
    if weight_out is None:
        weight_out = weight
    causal, scale = bool(causal), float(scale)
    key = ("attend", _sig(q), _sig(out), _sig(lse), _sig(weight), _sig(weight_out), _sig(row_counts), causal, scale, _sig(workspace))
    plan = cache.plans.get(key) or cache.plans.keep(
        key, _attend_plan(cache, q, out, lse, weight, weight_out, row_counts, causal, scale, workspace))
    _check(_load().kvc_attend(cache.ref, plan[0], q.data_ptr(), _ptr(row_counts), out.data_ptr(), _ptr(lse), _ptr(weight), _ptr(weight_out),
                              _ptr(workspace), plan[1], _launch_stream(plan[2], stream)))


def _evict_plan(src, dst, weight, budget, idx_out, weight_out):
    b, h = src.batch, src.n_kv_heads
    _dense(weight, "weight", torch.float32, b, h, src.capacity)
    _dense(idx_out, "idx_out", torch.int32, b, h, budget)
    _dense(weight_out, "weight_out", torch.float32, b, h, dst.capacity)
    return (_one_device(src.k, dst.k, weight, idx_out, weight_out),)


def kvc_evict(src: Cache, dst: Cache, weight: torch.Tensor, budget: int, recent: int, idx_out: torch.Tensor,
              weight_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """The last ``recent`` rows of every head and the heaviest of the others, ``budget`` in all, from src into dst; their
    positions go to idx_out [batch, Hkv, budget] int32, their weights to weight_out [batch, Hkv, dst.capacity]."""
    budget, recent = int(budget), int(recent)
    key = ("evict", dst.capacity, dst.k.get_device(), _sig(weight), budget, _sig(idx_out), _sig(weight_out))
    plan = src.plans.get(key) or src.plans.keep(key, _evict_plan(src, dst, weight, budget, idx_out, weight_out))
    _check(_load().kvc_evict(src.ref, dst.ref, weight.data_ptr(), budget, recent, idx_out.data_ptr(), _ptr(weight_out),
                             _launch_stream(plan[0], stream)))
