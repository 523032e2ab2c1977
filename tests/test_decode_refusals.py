"""What the decoding entry points refuse, found on the host before anything could launch (no GPU needed), and the plain
definitions that the GPU tests compare with, against torch's own conversions."""
import ctypes as C
import math

import pytest
import torch

import decode_ref as R
import paper_2509_05165_b200 as kvc
from paper_2509_05165_b200 import binding

BF = torch.bfloat16


def _cache(batch=2, heads=2, d=64, cap=100, block=32, dtype=torch.int8):
    return kvc.alloc_cache(batch, heads, d, cap, block, dtype, device="cpu")


def _refused(call, status=-1):
    with pytest.raises(kvc.KvcError) as e:
        call()
    # (these tensors are in host memory, which a machine with a GPU refuses before the library looks at the rest)
    assert e.value.status in ((status, -1) if torch.cuda.is_available() else (status,)), str(e.value)
    assert len(str(e.value)) > 10


def _struct(**kw):
    s = binding.KvcCache.from_buffer_copy(_cache().struct)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("field,value,status", [
    ("batch", 0, -1), ("n_kv_heads", 0, -1), ("batch", 40000, -2), ("head_dim", 96, -2), ("block", 48, -2), ("block", 256, -2),
    ("format", 2, -1), ("reserved_", 1, -1), ("capacity", 0, -1), ("capacity", 1 << 31, -2), ("k", None, -1), ("v_exp", None, -1),
    ("lengths", None, -1), ("k", 0x1008, -1), ("lengths", 0x1002, -1),
])
def test_bad_caches_are_refused(field, value, status):
    lib = binding._load()
    s = _struct(**{field: value})
    out = C.c_size_t(0)
    d = binding.KvcAttendDesc(4, 1, kvc.BF16, 1, 0.0, 0)
    assert lib.kvc_attend_workspace_size(C.byref(s), C.byref(d), 0, C.byref(out)) == status
    assert lib.kvc_cache_read(C.byref(s), None, 4, kvc.BF16, 0x1000, None, None) == status
    assert lib.kvc_cache_append(C.byref(s), 0x1000, 0x1000, kvc.BF16, 1, None, None, None, None, None, None) == status
    assert lib.kvc_evict(C.byref(s), C.byref(_struct()), 0x1000, 5, 1, 0x1000, None, None) == status
    assert lib.kvc_last_error()


def test_cache_strides_that_overlap_or_misalign_are_refused():
    lib = binding._load()
    for stride in ((6400, 6400, 64), (12800, 6400, 72), (12800, 6400, 32), (-12800, 6400, 64), (12800, 6399, 64)):
        s = _struct(stride=(C.c_int64 * 3)(*stride))
        assert lib.kvc_cache_read(C.byref(s), None, 4, kvc.BF16, 0x1000, None, None) == -1, stride


@pytest.mark.parametrize("field,value,status", [
    ("n_q_heads", 3, -1), ("n_q_heads", 0, -1), ("n_q_heads", 512, -2), ("rows", 0, -1), ("rows", 1 << 17, -2), ("dtype", 5, -1),
    ("causal", 2, -1), ("reserved_", 1, -1), ("scale", math.inf, -1), ("scale", math.nan, -1),
])
def test_bad_attention_descriptors_are_refused(field, value, status):
    lib = binding._load()
    d = binding.KvcAttendDesc(4, 1, kvc.BF16, 1, 0.0, 0)
    setattr(d, field, value)
    out = C.c_size_t(0)
    assert lib.kvc_attend_workspace_size(C.byref(_struct()), C.byref(d), 0, C.byref(out)) == status


def test_attention_arguments():
    c = _cache(dtype=torch.float8_e4m3fn)
    q = torch.zeros((2, 4, 1, 64), dtype=BF)
    need = kvc.kvc_attend_workspace_size(c, q, True)
    assert 0 < kvc.kvc_attend_workspace_size(c, q, False) <= need and need % 256 == 0
    _refused(lambda: kvc.kvc_attend(c, q, q.clone()), -3)                                        # no workspace
    _refused(lambda: kvc.kvc_attend(c, q, q.clone(), workspace=torch.zeros(256, dtype=torch.uint8)[1:]), -3)
    _refused(lambda: kvc.kvc_attend(c, q, q.float()))                                            # another type
    _refused(lambda: kvc.kvc_attend(c, q.half(), q.half()))
    _refused(lambda: kvc.kvc_attend(c, q[:1], q[:1]))                                            # another batch
    _refused(lambda: kvc.kvc_attend(c, q, q.expand(2, 4, 3, 64)))
    _refused(lambda: kvc.kvc_attend(c, q, q.clone(), weight=torch.zeros(2, 2, 99)))
    _refused(lambda: kvc.kvc_attend(c, q, q.clone(), lse=torch.zeros(2, 4)))
    _refused(lambda: kvc.kvc_attend(c, q, q.clone(), row_counts=torch.zeros(2)))
    many = torch.zeros((2, 4, 3, 64), dtype=BF)
    _refused(lambda: kvc.kvc_attend(c, many, torch.zeros((2, 4, 1, 64), dtype=BF).expand(2, 4, 3, 64), workspace=torch.zeros(need)))
    lib = binding._load()
    d = binding.KvcAttendDesc(4, 1, kvc.BF16, 1, 0.0, 0)
    assert lib.kvc_attend(C.byref(c.struct), C.byref(d), 0x1000, None, 0x1000, None, 0x1000, None, 0x1000, 1 << 30, None) == -1
    assert lib.kvc_attend(C.byref(c.struct), C.byref(d), 0x1008, None, 0x1000, None, None, None, 0x1000, 1 << 30, None) == -1
    assert lib.kvc_attend(C.byref(c.struct), C.byref(d), None, None, 0x1000, None, None, None, 0x1000, 1 << 30, None) == -1


def test_cache_tensors_of_the_wrong_kind():
    c = _cache()
    ok = (c.k, c.v, c.k_exp, c.v_exp, c.lengths)
    kvc.Cache(*ok, 32)
    _refused(lambda: kvc.Cache(c.k.float(), *ok[1:], 32))
    _refused(lambda: kvc.Cache(*ok, 64))                                # another number of exponents
    _refused(lambda: kvc.Cache(*ok, 20))
    _refused(lambda: kvc.Cache(c.k, c.v[:, :, :99], *ok[2:], 32))
    _refused(lambda: kvc.Cache(c.k, c.v.transpose(0, 1).contiguous().transpose(0, 1), *ok[2:], 32))
    _refused(lambda: kvc.Cache(c.k, c.v, c.k_exp, c.v_exp, c.lengths.long(), 32))
    _refused(lambda: kvc.Cache(c.k.transpose(2, 3), c.v.transpose(2, 3), *ok[2:], 32))


def test_gather_append_and_read_arguments():
    c = _cache()
    d = kvc.kvc_desc_init(1, 2, 4, 2, 64, 50, 1, kvc.BF16)
    k = [torch.zeros((2, 2, 50, 64), dtype=BF)]
    _refused(lambda: kvc.kvc_cache_gather(d, k, k, None, None, [c, c]))
    _refused(lambda: kvc.kvc_cache_gather(d, [k[0].float()], k, None, None, [c]))
    _refused(lambda: kvc.kvc_cache_gather(d, k, k, torch.zeros((1, 2, 2, 49), dtype=torch.int32), None, [c]))
    _refused(lambda: kvc.kvc_cache_gather(d, k, k, None, torch.zeros((2, 1), dtype=torch.int32), [c], per_head=True))
    _refused(lambda: kvc.kvc_cache_gather(d, k, k, None, None, [_cache(heads=1)]))
    _refused(lambda: kvc.kvc_cache_gather(d, [k[0].transpose(0, 1).contiguous().transpose(0, 1)], k, None, None, [c]))
    two = kvc.kvc_desc_init(2, 2, 4, 2, 64, 50, 1, kvc.BF16)
    _refused(lambda: kvc.kvc_cache_gather(two, k * 2, k * 2, None, None, [c, _cache(block=16)]))
    x = k[0]
    _refused(lambda: kvc.kvc_cache_append(c, x.half(), x.half()))
    _refused(lambda: kvc.kvc_cache_append(c, x, x[:, :, :49]))
    _refused(lambda: kvc.kvc_cache_append(c, x, x.float()))
    _refused(lambda: kvc.kvc_cache_append(c, x[:, :, :0], x[:, :, :0]))
    _refused(lambda: kvc.kvc_cache_append(c, x, x, n_new=torch.zeros(3, dtype=torch.int32)))
    _refused(lambda: kvc.kvc_cache_append(c, x, x, weight=torch.zeros(2, 2, 50)))
    _refused(lambda: kvc.kvc_cache_append(c, x, x, lengths_out=torch.zeros((2, 2))))
    _refused(lambda: kvc.kvc_cache_read(c, None, None))
    _refused(lambda: kvc.kvc_cache_read(c, x, x.float()))
    _refused(lambda: kvc.kvc_cache_read(c, x.transpose(0, 1), None))
    _refused(lambda: kvc.kvc_cache_read(c, x, None, first=torch.zeros((2, 2), dtype=torch.int64)))


def test_eviction_arguments():
    a, b = _cache(), _cache(cap=40)
    w = torch.zeros((2, 2, 100))
    idx = lambda n: torch.zeros((2, 2, n), dtype=torch.int32)  # noqa: E731
    _refused(lambda: kvc.kvc_evict(a, b, w, 41, 0, idx(41)))
    _refused(lambda: kvc.kvc_evict(a, b, w, 0, 0, idx(0)))
    _refused(lambda: kvc.kvc_evict(a, b, w, 40, 41, idx(40)))
    _refused(lambda: kvc.kvc_evict(a, b, w, 40, -1, idx(40)))
    _refused(lambda: kvc.kvc_evict(a, a, w, 40, 4, idx(40)))
    _refused(lambda: kvc.kvc_evict(a, b, w, 40, 4, idx(39)))
    _refused(lambda: kvc.kvc_evict(a, _cache(cap=40, dtype=torch.float8_e4m3fn), w, 40, 4, idx(40)))
    _refused(lambda: kvc.kvc_evict(a, _cache(), w, 40, 4, idx(40), weight_out=w))
    _refused(lambda: kvc.kvc_evict(a, kvc.Cache(b.k, b.v, b.k_exp, b.v_exp, a.lengths, 32), w, 40, 4, idx(40)))
    _refused(lambda: kvc.kvc_evict(a, kvc.Cache(b.k, b.v, b.k_exp, a.k_exp.view(-1)[:8].view(2, 2, 2), b.lengths, 32), w, 40, 4, idx(40)))


def _rope(**kw):
    return kvc.Rotary(**dict(dict(rot_dim=64), **kw))


def test_rotary_arguments():
    q, pos = torch.zeros((2, 4, 3, 64), dtype=BF), torch.arange(3)
    for kw, status in ((dict(rot_dim=24), -2), (dict(rot_dim=80), -2), (dict(rot_dim=0), -2), (dict(theta=1.0), -1), (dict(theta=math.inf), -1),
                       (dict(scaling="linear", factor=0.5), -1), (dict(scaling="cubic"), -1),
                       (dict(scaling="banded", factor=8.0, turns_low=4.0, turns_high=4.0), -1),
                       (dict(scaling="yarn", factor=8.0, turns_low=0.0), -1), (dict(scaling="yarn", factor=8.0, original_ctx=0.0), -1),
                       (dict(mscale=-1.0), -1), (dict(mscale=math.nan), -1)):
        _refused(lambda: kvc.kvc_rotary(_rope(**kw), q, None, pos), status)
    _refused(lambda: kvc.kvc_rotary(_rope(), None, None, pos))
    _refused(lambda: kvc.kvc_rotary(_rope(), q, None, pos.int()))
    _refused(lambda: kvc.kvc_rotary(_rope(), q, None, torch.arange(4)))
    _refused(lambda: kvc.kvc_rotary(_rope(), q, q.float(), pos))
    _refused(lambda: kvc.kvc_rotary(_rope(), q, None, pos, q[:, :2]))
    _refused(lambda: kvc.kvc_rotary(_rope(), q, None, pos, None, q))
    _refused(lambda: kvc.kvc_rotary(_rope(), q, None, pos, torch.zeros((2, 1, 3, 64), dtype=BF).expand(2, 4, 3, 64)))   # heads on one another
    _refused(lambda: kvc.kvc_rotary(_rope(), torch.zeros((2, 4, 3, 68), dtype=BF)[..., 4:], None, pos))                # rows on 8 bytes


# ---- the definitions ---------------------------------------------------------------------------------------------------

def test_the_definition_of_an_exponent_at_its_borders():
    for dt, q in R.QMAX.items():
        for k in (-90, -1, 0, 1, 100):
            assert R.exponent(math.ldexp(q, k), dt) == k
            assert R.exponent(math.nextafter(math.ldexp(q, k), math.inf), dt) == k + 1
            assert R.exponent(math.nextafter(math.ldexp(q, k), 0.0), dt) == k
        assert R.exponent(0.0, dt) == R.exponent(1e-45, dt) == -100
        assert R.exponent(math.inf, dt) == 121


def test_the_definition_of_a_code_is_torchs_rounding():
    g = torch.Generator().manual_seed(0)
    x = torch.cat([torch.randn(20000, generator=g) * 100, torch.randn(20000, generator=g) * 0.02, torch.arange(-448, 448.25, 0.25)]).clamp(-448, 448)
    want = x.to(torch.float8_e4m3fn).double()
    assert torch.equal(R.round_code(x.double(), torch.float8_e4m3fn), want)
    y = x.clamp(-127, 127)
    assert torch.equal(R.round_code(y.double(), torch.int8), torch.round(y).double())


def test_a_row_that_moves_keeps_its_code_unless_the_exponent_grows():
    for dt in R.QMAX:
        h = R.Held(dt, 16).fill(torch.randn(16, 8, generator=torch.Generator().manual_seed(1)))
        v = h.values()
        assert torch.equal(R.Held(dt, 16).fill(v).values(), v)
