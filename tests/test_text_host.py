"""CPU-only checks of the text operators' argument checks: every refusal is found on the host, before any launch."""
import os

import pytest
import torch

from paper_2604_08077_b200 import binding, build


@pytest.fixture(scope="module")
def handle():
    build.build()
    h = binding.adaspark_attn_create(binding.Config(4, 4, 4, 28, 4, 128, 0.9, 0.0, 0, 0))
    yield h
    binding.adaspark_attn_destroy(h)


P = 1 << 20                                   # a pointer that is never followed
ROW = (P, 0, 0)


def pages(**kw):
    f = dict(k_pages=P, v_pages=P, k_scale=P, v_scale=P, page_stride=0, scale_stride=0, n_pages=8, page_size=16, format=binding.PAGES_E4M3, reserved=0)
    f.update(kw)
    f.pop("reserved")
    f["page_format"] = f.pop("format")
    return binding.pages_struct(**f)


def code(fn, *a):
    with pytest.raises(binding.AdasparkError) as e:
        fn(*a)
    return e.value.status


def prompt(handle, **kw):
    f = dict(q=ROW, k=ROW, v=ROW, cu_q=P, cu_k=P, batch=2, n_q=10, n_k=10, out=P, lse=None, ws=P, ws_bytes=binding.adaspark_attn_text_workspace_bytes(handle), status=None)
    f.update(kw)
    binding.adaspark_attn_prompt(handle, *f.values(), None)


def test_workspace_size_is_known_without_a_partition(handle):
    n = binding.adaspark_attn_text_workspace_bytes(handle)
    assert n > 0 and n % 256 == 0
    assert binding.load().adaspark_attn_text_workspace_bytes(None) == 0


@pytest.mark.parametrize("bad,status", [
    (dict(q=(0, 0, 0)), binding.ERR_INVALID_ARG), (dict(k=(0, 0, 0)), binding.ERR_INVALID_ARG), (dict(out=None), binding.ERR_INVALID_ARG),
    (dict(cu_q=None), binding.ERR_INVALID_ARG), (dict(cu_k=None), binding.ERR_INVALID_ARG), (dict(batch=-1), binding.ERR_INVALID_ARG),
    (dict(n_q=-1), binding.ERR_INVALID_ARG), (dict(n_k=-4), binding.ERR_INVALID_ARG), (dict(q=(P + 8, 0, 0)), binding.ERR_INVALID_ARG),
    (dict(v=(P, 130, 0)), binding.ERR_INVALID_ARG), (dict(k=(P, 0, 64)), binding.ERR_INVALID_ARG), (dict(q=(P, -256, 0)), binding.ERR_INVALID_ARG),
    (dict(out=P + 2), binding.ERR_INVALID_ARG), (dict(ws=None), binding.ERR_INVALID_ARG), (dict(ws=P + 16), binding.ERR_INVALID_ARG),
    (dict(ws_bytes=0), binding.ERR_WORKSPACE_TOO_SMALL)])
def test_prompt_refusals(handle, bad, status):
    assert code(lambda: prompt(handle, **bad)) == status
    assert binding.load().adaspark_attn_last_error(handle)


def test_nothing_to_do_is_no_error(handle):
    prompt(handle, batch=0)
    prompt(handle, n_q=0, q=(0, 0, 0))
    assert binding.adaspark_attn_last_launch_count(handle) == 0
    binding.adaspark_attn_paged_write(handle, pages(), ROW, ROW, P, 2, 0, P, 4, P, None, None)
    binding.adaspark_attn_paged_read(handle, pages(), ROW, ROW, P, 0, 5, P, 4, P, None, None)
    binding.adaspark_attn_paged_decode(handle, ROW, (0, 0, 0), (0, 0, 0), pages(), P, 4, P, 0, P, None, P, 0, None, None)


@pytest.mark.parametrize("bad,status", [
    (dict(page_size=24), binding.ERR_UNSUPPORTED), (dict(page_size=8), binding.ERR_UNSUPPORTED), (dict(page_size=512), binding.ERR_UNSUPPORTED),
    (dict(format=7), binding.ERR_UNSUPPORTED), (dict(n_pages=0), binding.ERR_INVALID_ARG), (dict(k_pages=None), binding.ERR_INVALID_ARG),
    (dict(v_scale=None), binding.ERR_INVALID_ARG), (dict(k_pages=P + 8), binding.ERR_INVALID_ARG), (dict(page_stride=4 * 16 * 128 - 16), binding.ERR_INVALID_ARG),
    (dict(page_stride=4 * 16 * 128 + 8), binding.ERR_INVALID_ARG), (dict(scale_stride=72), binding.ERR_INVALID_ARG), (dict(scale_stride=48), binding.ERR_INVALID_ARG)])
def test_page_refusals(handle, bad, status):
    p = pages(**bad)
    ws = binding.adaspark_attn_text_workspace_bytes(handle)
    assert code(binding.adaspark_attn_paged_write, handle, p, ROW, ROW, P, 2, 5, P, 4, P, None, None) == status
    assert code(binding.adaspark_attn_paged_read, handle, p, ROW, ROW, P, 2, 5, P, 4, P, None, None) == status
    assert code(binding.adaspark_attn_paged_decode, handle, ROW, ROW, ROW, p, P, 4, P, 2, P, None, P, ws, None, None) == status


def test_packed_structs_are_the_headers(tmp_path):
    """The sizes that the binding packs are the compiler's."""
    import subprocess
    src = tmp_path / "sizes.c"
    names = ["adaspark_attn_pages_t", "adaspark_attn_prompt_t", "adaspark_attn_paged_rows_t", "adaspark_attn_paged_decode_t"]
    src.write_text('#include "adaspark_attn.h"\n#include <stdio.h>\nint main(void) { printf("' + "%zu " * 4 + '", ' + ", ".join(f"sizeof({n})" for n in names) + "); return 0; }")
    subprocess.run(["gcc", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include"), "-o", str(tmp_path / "sizes"), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()]
    p = binding._PAGES.size
    assert got == [p, binding._PROMPT.size, p + binding._PAGED_ROWS.size, p + binding._PAGED_DECODE.size]


def test_other_paged_refusals(handle):
    ws = binding.adaspark_attn_text_workspace_bytes(handle)
    none = (0, 0, 0)
    dec = binding.adaspark_attn_paged_decode
    assert code(dec, handle, ROW, ROW, none, pages(), P, 4, P, 2, P, None, P, ws, None, None) == binding.ERR_INVALID_ARG
    assert code(dec, handle, none, none, none, pages(), P, 4, P, 2, P, None, P, ws, None, None) == binding.ERR_INVALID_ARG
    assert code(dec, handle, ROW, none, none, pages(), P, 4, None, 2, P, None, P, ws, None, None) == binding.ERR_INVALID_ARG
    assert code(dec, handle, ROW, none, none, pages(), P, 0, P, 2, P, None, P, ws, None, None) == binding.ERR_INVALID_ARG
    assert code(dec, handle, ROW, none, none, pages(page_size=256), P, 1 << 23, P, 2, P, None, P, ws, None, None) == binding.ERR_UNSUPPORTED
    assert code(dec, handle, ROW, none, none, pages(), P, 4, P, 2, P, None, P, ws - 1, None, None) == binding.ERR_WORKSPACE_TOO_SMALL
    assert code(dec, handle, ROW, none, none, pages(), P, 4, P, -2, P, None, P, ws, None, None) == binding.ERR_INVALID_ARG
    assert code(binding.adaspark_attn_paged_write, handle, pages(), ROW, ROW, None, 2, 5, P, 4, P, None, None) == binding.ERR_INVALID_ARG
    assert code(binding.adaspark_attn_paged_write, handle, pages(), ROW, ROW, P, 2, 5, None, 4, P, None, None) == binding.ERR_INVALID_ARG
    assert code(binding.adaspark_attn_paged_read, handle, pages(), ROW, (P + 4, 0, 0), P, 2, 5, P, 4, P, None, None) == binding.ERR_INVALID_ARG
    for name in ("prompt", "paged_write", "paged_read", "paged_decode"):
        assert getattr(binding.load(), "adaspark_attn_" + name)(None, b"", None) == binding.ERR_INVALID_ARG
        assert getattr(binding.load(), "adaspark_attn_" + name)(handle, None, None) == binding.ERR_INVALID_ARG


def test_without_a_gpu_the_calls_fail_loudly(handle):
    if torch.cuda.is_available():
        pytest.skip("a GPU is there")
    assert code(lambda: prompt(handle)) == binding.ERR_CUDA


def test_paged_cache_refusals():
    k = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    refused = lambda *a: code(binding.PagedCache, *a) == binding.ERR_INVALID_ARG  # noqa: E731
    s = torch.zeros(3, 2, 16, dtype=torch.uint8)
    q = k.to(torch.float8_e4m3fn)
    assert refused(k, k[:2]) and refused(k.half(), k.half()) and refused(k[0], k[0]) and refused(k, k, s, s)
    assert refused(q, q) and refused(q, q, s, s[:2]) and refused(q, q, s, s.to(torch.int32))
    assert refused(k.transpose(1, 2), k.transpose(1, 2)) and refused(k[:0], k[:0])
    pool = torch.zeros(6, 2, 16, 64, dtype=torch.bfloat16)
    assert refused(pool[::2], k)
    c = binding.PagedCache(pool[::2], pool[1::2])                # keys and values of a page beside each other
    assert c.page_stride == 2 * 2 * 16 * 64 and c.n_pages == 3 and c.page_size == 16
    assert binding.PagedCache(q, q.clone(), s, s.clone()).pages[-8:] == binding.PAGES_E4M3.to_bytes(8, "little")
