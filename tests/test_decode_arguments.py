"""What the decoding calls keep between calls, and what they hand to the library, found on the host (no GPU needed)."""
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
