"""Copies of the objects that hold addresses: a copy's are those of its own memory, also where the original is gone or in another process."""
import copy
import ctypes
import io
import pickle
import struct

import pytest
import torch

from paper_2604_08077_b200 import binding


@pytest.mark.parametrize("again", [copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r))])
def test_rotary(again):
    r = binding.Rotary(128, sections=[16, 24, 24], theta=1e6, adjacent=True)
    c = again(r)
    assert c.address == ctypes.addressof(c.struct) and bytes(c.struct) == bytes(r.struct)
    assert (c.axes, c.pairs, c.head_dim) == (3, 64, 128)
    assert again is copy.copy or c.address != r.address


def saved_and_loaded(x):
    f = io.BytesIO()
    torch.save(x, f)
    f.seek(0)
    return torch.load(f, weights_only=False)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("again", [copy.copy, copy.deepcopy, saved_and_loaded])
def test_paged_cache(again, e4m3):
    pool = torch.zeros(2, 8, 2, 16, 64, dtype=torch.bfloat16)
    tensors = [pool[0, ::2], pool[1, ::2]]
    if e4m3:
        tensors = [torch.zeros(4, 2, 16, 64, dtype=torch.float8_e4m3fn) for _ in range(2)] + [torch.zeros(4, 2, 16, dtype=torch.uint8) for _ in range(2)]
    cache = binding.PagedCache(*tensors)
    c = again(cache)
    held = [c.k_pages, c.v_pages, c.k_scale, c.v_scale]
    assert list(struct.unpack_from("4Q", c.pages)) == [0 if t is None else t.data_ptr() for t in held]
    assert (c.n_pages, c.page_size, c.n_kv_heads, c.head_dim, c.device) == (4, 16, 2, 64, cache.device)
    assert struct.unpack_from("2q", c.pages, 32)[0] == c.page_stride and (c.page_stride == c.k_pages.stride(0))
    if again is not copy.copy:
        assert c.k_pages.data_ptr() != cache.k_pages.data_ptr()
