"""CPU-only checks of what rotated positions, appending and chunks over pages refuse, and of the fixed-point angles."""
import ctypes
import math
import os
import subprocess
from fractions import Fraction

import pytest
import torch

from paper_2604_08077_b200 import binding, build

P = 1 << 20                                   # a pointer that is never followed
ROW, NONE = (P, 0, 0), (0, 0, 0)
INVALID, UNSUPPORTED = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def handle():
    build.build()
    h = binding.adaspark_attn_create(binding.Config(4, 4, 4, 28, 4, 128, 0.9, 0.0, 0, 0))
    yield h
    binding.adaspark_attn_destroy(h)


def code(fn, *a):
    with pytest.raises(binding.AdasparkError) as e:
        fn(*a)
    return e.value.status


def pages(**kw):
    f = dict(k_pages=P, v_pages=P, k_scale=P, v_scale=P, page_stride=0, scale_stride=0, n_pages=8, page_size=16, page_format=binding.PAGES_E4M3)
    f.update(kw)
    return binding.pages_struct(**f)


def rotate(handle, **kw):
    f = dict(q=ROW, k=ROW, q_out=ROW, k_out=ROW, positions=P, rotary=binding.Rotary(128).address, q_norm=None, k_norm=None, eps=1e-6, n=5)
    f.update(kw)
    binding.adaspark_attn_rotate(handle, *f.values(), None)


def append(handle, **kw):
    f = dict(q=ROW, k=ROW, v=ROW, q_out=ROW, pages=pages(), cu=P, batch=2, n=5, block_table=P, table_width=4, kv_len=P, positions=None, rotary=None, q_norm=None,
             k_norm=None, eps=0.0, status=None)
    f.update(kw)
    binding.adaspark_attn_paged_append(handle, *f.values(), None)


def chunk(handle, **kw):
    f = dict(q=ROW, pages=pages(), cu=P, batch=2, n=5, block_table=P, table_width=4, kv_len=P, window=0, sinks=0, out=P, lse=None, ws=P,
             ws_bytes=binding.adaspark_attn_text_workspace_bytes(handle), status=None)
    f.update(kw)
    binding.adaspark_attn_paged_prompt(handle, *f.values(), None)


def decode(handle, **kw):
    f = dict(q=ROW, k_new=NONE, v_new=NONE, pages=pages(), block_table=P, table_width=4, kv_len=P, batch=2, out=P, lse=None, ws=P,
             ws_bytes=binding.adaspark_attn_text_workspace_bytes(handle), status=None, window=5, sinks=0)
    f.update(kw)
    binding.adaspark_attn_paged_decode_window(handle, *f.values(), None)


def test_packed_structs_are_the_headers(tmp_path):
    names = ["adaspark_attn_paged_decode_window_t", "adaspark_attn_paged_prompt_t", "adaspark_attn_rotary_t", "adaspark_attn_rotate_t", "adaspark_attn_paged_append_t"]
    src = tmp_path / "sizes.c"
    src.write_text('#include "adaspark_attn.h"\n#include <stdio.h>\nint main(void) { printf("' + "%zu " * 5 + '", ' + ", ".join(f"sizeof({n})" for n in names) + "); return 0; }")
    subprocess.run(["gcc", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include"), "-o", str(tmp_path / "sizes"), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()]
    p = binding._PAGES.size
    assert got == [p + binding._PAGED_DECODE.size + binding._WINDOW.size, p + binding._PAGED_PROMPT.size, ctypes.sizeof(binding.RotaryStruct), binding._ROTATE.size,
                   p + binding._PAGED_APPEND.size]


def test_angles_are_fractions_of_a_turn():
    """turns[i] is radians / 2 pi modulo 1 as 64-bit fixed point: within 2^-52 of a turn of the exact one (the frequency is a double), for every sign and size."""
    two_pi = Fraction("6.283185307179586476925286766559005768394338798750211641949889")
    radians = [1.0, 1e-6, 1e-9, 0.0, -1.0, -1e-7, 6.283185307179586, 100.25]
    r = binding.adaspark_attn_rotary_init(radians, None, 1, False)
    for x, got in zip(radians, r.turns):
        turns = Fraction(x) / two_pi
        off = (Fraction(got, 2 ** 64) - turns) % 1
        off = min(off, 1 - off)
        assert off <= max(abs(turns), 1) * Fraction(1, 2 ** 62), x
    assert (r.pairs, r.axes, r.adjacent, list(r.axis[:8])) == (8, 1, 0, [0] * 8)
    assert binding.Rotary(64, sections=[8, 12, 12]).axes == 3
    r = binding.Rotary(128, sections=[16, 24, 24], theta=1e6)
    assert list(r.struct.axis) == [0] * 16 + [1] * 24 + [2] * 24
    assert math.isclose(r.struct.turns[63] / 2 ** 64, 1e6 ** (-63 / 64) / (2 * math.pi), rel_tol=1e-12)


def test_rotary_refusals(handle):
    init = binding.adaspark_attn_rotary_init
    assert code(init, [1.0] * 7, None, 1, False) == INVALID and code(init, [1.0] * 72, None, 1, False) == INVALID
    assert code(init, [1.0] * 7 + [math.inf], None, 1, False) == INVALID and code(init, [math.nan] * 8, None, 1, False) == INVALID
    assert code(init, [1.0] * 8, [0] * 7 + [3], 3, False) == INVALID and code(init, [1.0] * 8, [-1] * 8, 3, False) == INVALID
    assert code(init, [1.0] * 8, None, 0, False) == INVALID and code(init, [1.0] * 8, None, 300, False) == INVALID
    assert binding.load().adaspark_attn_rotary_init(None, None, None, 0, 1, 0) == INVALID
    assert init([], None, 1, False).pairs == 0
    for kw in (dict(sections=[40]), dict(sections=[]), dict(sections=[-8, 16]), dict(theta=0.0), dict(axis=[0] * 32), dict(frequencies=[1.0] * 8, sections=[8]),
               dict(frequencies=[1.0] * 8, axis=[0] * 7), dict(frequencies=[1.0] * 40)):
        assert code(lambda: binding.Rotary(64, **kw)) == INVALID, kw


@pytest.mark.parametrize("bad", [dict(q=(P + 8, 0, 0)), dict(q_out=NONE), dict(k_out=NONE), dict(k_out=(P, 64, 0)), dict(q=(P, 0, 12)), dict(positions=None), dict(eps=-1.0),
                                 dict(eps=math.nan), dict(eps=math.inf), dict(q_norm=P + 2), dict(k_norm=P + 8), dict(n=-1)])
def test_rotate_refusals(handle, bad):
    assert code(lambda: rotate(handle, **bad)) == INVALID
    assert binding.load().adaspark_attn_last_error(handle)


def test_rotations_that_do_not_fit(handle):
    small = binding.adaspark_attn_create(binding.Config(4, 4, 4, 4, 4, 64, 0.9, 0.0, 0, 0))
    assert code(lambda: rotate(small)) == INVALID              # 64 pairs in a head of 64
    binding.adaspark_attn_destroy(small)
    r = binding.Rotary(128)
    r.struct.axis[5] = 1
    assert code(lambda: rotate(handle, rotary=r.address)) == INVALID
    r.struct.axis[5], r.struct.pairs = 0, 12
    assert code(lambda: append(handle, rotary=r.address)) == INVALID


@pytest.mark.parametrize("bad,status", [
    (dict(k=NONE), INVALID), (dict(v=NONE), INVALID), (dict(q_out=NONE), INVALID), (dict(cu=None), INVALID), (dict(kv_len=None), INVALID), (dict(block_table=None), INVALID),
    (dict(batch=-1), INVALID), (dict(n=-2), INVALID), (dict(table_width=0), INVALID), (dict(pages=pages(page_size=48)), UNSUPPORTED), (dict(eps=-0.5), INVALID),
    (dict(pages=pages(v_scale=None)), INVALID)])
def test_append_refusals(handle, bad, status):
    assert code(lambda: append(handle, **bad)) == status


@pytest.mark.parametrize("call", [chunk, decode])
@pytest.mark.parametrize("bad,status", [
    (dict(q=NONE), INVALID), (dict(kv_len=None), INVALID), (dict(block_table=None), INVALID), (dict(out=None), INVALID), (dict(out=P + 4), INVALID), (dict(ws=None), INVALID),
    (dict(ws_bytes=0), binding.ERR_WORKSPACE_TOO_SMALL), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(batch=-1), INVALID), (dict(table_width=0), INVALID),
    (dict(pages=pages(page_format=3)), UNSUPPORTED), (dict(pages=pages(n_pages=0)), INVALID)])
def test_attention_refusals(handle, call, bad, status):
    assert code(lambda: call(handle, **bad)) == status


def test_other_refusals(handle):
    assert code(lambda: chunk(handle, cu=None)) == INVALID and code(lambda: chunk(handle, n=-1)) == INVALID
    assert code(lambda: chunk(handle, table_width=(1 << 27) - 1, window=7)) == UNSUPPORTED
    assert code(lambda: decode(handle, window=0)) == INVALID and code(lambda: decode(handle, k_new=ROW)) == INVALID
    for name in ("paged_decode_window", "paged_prompt", "rotate", "paged_append"):
        assert getattr(binding.load(), "adaspark_attn_" + name)(None, b"", None) == INVALID
        assert getattr(binding.load(), "adaspark_attn_" + name)(handle, None, None) == INVALID


def test_nothing_to_do_is_no_error(handle):
    rotate(handle, n=0)
    rotate(handle, q=NONE, k=NONE)
    append(handle, n=0)
    append(handle, batch=0)
    chunk(handle, batch=0)
    chunk(handle, n=0)
    decode(handle, batch=0)
    assert binding.adaspark_attn_last_launch_count(handle) == 0


def test_without_a_gpu_the_calls_fail_loudly(handle):
    if torch.cuda.is_available():
        pytest.skip("a GPU is there")
    for call in (rotate, append, chunk, decode):
        assert code(lambda: call(handle)) == binding.ERR_CUDA
