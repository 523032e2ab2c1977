"""What the decoding calls keep between calls, and what they hand to the library, found on the host (no GPU needed)."""
import copy
import copy
import math
import pickle

import pytest
import torch

import paper_2509_05165_b200 as kvc

BF = torch.bfloat16


def _status(call):
    with pytest.raises(kvc.KvcError) as e:
        call()
    return e.value.status


def _cache(cap=100):
    return kvc.alloc_cache(2, 2, 64, cap, 32, torch.int8, device="cpu")


def test_a_workspace_of_repeated_bytes_is_refused():
    """Its size in elements says nothing about the memory behind it."""
    c, q = _cache(), torch.zeros((2, 4, 1, 64), dtype=BF)
    need = kvc.kvc_attend_workspace_size(c, q, False)
    store = torch.zeros(512, dtype=torch.uint8)
    at = -store.data_ptr() % 256
    assert _status(lambda: kvc.kvc_attend(c, q, q.clone(), workspace=store[at:at + 1].expand(need))) == -1
    wide = torch.zeros((need // 256 + 1, 512), dtype=torch.uint8)
    assert _status(lambda: kvc.kvc_attend(c, q, q.clone(), workspace=wide[:, :256])) == -1


def test_options_go_by_their_values():
    """A number in a tensor that changes between two calls: the second call is checked and made with what it holds then."""
    c, q = _cache(), torch.zeros((2, 4, 1, 64), dtype=BF)
    store = torch.zeros(kvc.kvc_attend_workspace_size(c, q, False) + 256, dtype=torch.uint8)
    ws = store[-store.data_ptr() % 256:]
    scale = torch.tensor(0.5)
    gpu = torch.cuda.is_available()
    first = _status(lambda: kvc.kvc_attend(c, q, q.clone(), scale=scale, workspace=ws))
    assert first == (-1 if gpu else -4)                     # (host tensors, or no device: past the checks)
    scale.fill_(math.nan)
    assert _status(lambda: kvc.kvc_attend(c, q, q.clone(), scale=scale, workspace=ws)) == -1
    dst, w, idx = _cache(60), torch.zeros((2, 2, 100)), torch.zeros((2, 2, 40), dtype=torch.int32)
    budget = torch.tensor(40)
    assert _status(lambda: kvc.kvc_evict(c, dst, w, budget, 4, idx)) == first
    budget.fill_(50)                                        # idx has no room for as many
    assert _status(lambda: kvc.kvc_evict(c, dst, w, budget, 4, idx)) == -1


def test_rotary_positions_are_copied_and_pickled():
    """As part of a model that is copied or sent to another process; the copy turns by the same frequencies, with plans of its own."""
    rope = kvc.Rotary(64, theta=500000.0, scaling="yarn", factor=16.0, turns_high=32.0, original_ctx=4096.0)
    q, pos = torch.zeros((1, 2, 3, 64), dtype=BF), torch.arange(3)
    _status(lambda: kvc.kvc_rotary(rope, q, None, pos))                    # (a plan is kept)
    for other in (copy.copy(rope), copy.deepcopy({"a": [rope]})["a"][0], pickle.loads(pickle.dumps(rope))):
        assert other == rope and hash(other) == hash(rope) and other is not rope
        assert bytes(other.struct) == bytes(rope.struct) and other.plans is not rope.plans and not other.plans
        assert _status(lambda: kvc.kvc_rotary(other, q, None, pos)) == _status(lambda: kvc.kvc_rotary(rope, q, None, pos))
