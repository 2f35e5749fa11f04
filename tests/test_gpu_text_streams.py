"""GPU tests of the text calls on a stream that is not torch's current one: what they report, and the memory that they allocate."""
import gc

import pytest
import torch

import text_util as tu
from paper_2604_08077_b200 import binding

pytestmark = pytest.mark.gpu

HQ, HKV, D, PAGE = 4, 2, 64, 16


def draw(g, *shape):
    return torch.randn(*shape, generator=g).to(torch.bfloat16).cuda()


def busy(stream=None):
    """About 0.1 s of nothing on a stream."""
    with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
        torch.cuda._sleep(200_000_000)


def bad_write(eng, g):
    """A write whose page number is out of range."""
    cache = eng.paged_cache(4, PAGE)
    k, v, cu = draw(g, 3, HKV, D), draw(g, 3, HKV, D), tu.cumulative([3])
    table, kv_len = torch.full((1, 1), 9, dtype=torch.int32, device="cuda"), torch.full((1,), 3, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    return lambda **kw: eng.paged_write(cache, k, v, cu, table, kv_len, **kw)


@pytest.mark.parametrize("by_argument", [True, False])
def test_status_waits_for_calls_on_other_streams(by_argument):
    eng, s = tu.engine(HQ, HKV, D), torch.cuda.Stream()
    call = bad_write(eng, torch.Generator().manual_seed(210))
    call()
    assert eng.text_status() == 1 and eng.text_status() == 0
    busy(s)
    if by_argument:
        call(stream=s)
    else:
        with torch.cuda.stream(s):
            call()
    assert eng.text_status() == 1 and eng.text_status() == 0


def test_status_of_a_first_call_on_another_stream():
    """What the first call sets up does not come after what it reports."""
    eng, s = tu.engine(HQ, HKV, D), torch.cuda.Stream()
    call = bad_write(eng, torch.Generator().manual_seed(211))
    busy()
    call(stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert eng.text_status() == 1


def test_status_inside_a_capture_is_refused():
    eng = tu.engine(HQ, HKV, D)
    bad_write(eng, torch.Generator().manual_seed(212))()
    g, x = torch.cuda.CUDAGraph(), torch.zeros(1, device="cuda")
    with torch.cuda.graph(g):
        x.add_(1)
        with pytest.raises(binding.AdasparkError):
            eng.text_status()
    assert eng.text_status() == 1


def prompt_call(g, n=700):
    eng, cu = tu.engine(HQ, HKV, D), tu.cumulative([n])
    q, k, v = draw(g, n, HQ, D), draw(g, n, HKV, D), draw(g, n, HKV, D)
    return eng, (n, HQ, D), lambda **kw: eng.prompt(q, k, v, cu, want_lse=True, **kw)


def decode_call(g, n=4000, B=300):
    """Cut over many runs, so that the workspace is used."""
    eng = tu.engine(HQ, HKV, D)
    cache = eng.paged_cache(n // PAGE + 1, PAGE)
    cache.k_pages.copy_(draw(g, *cache.k_pages.shape)), cache.v_pages.copy_(draw(g, *cache.v_pages.shape))
    table = torch.arange(n // PAGE + 1, dtype=torch.int32, device="cuda").repeat(B, 1)
    q, kv_len = draw(g, B, HQ, D), torch.full((B,), n, dtype=torch.int32, device="cuda")
    return eng, (B, HQ, D), lambda **kw: eng.paged_decode(q, None, None, cache, table, kv_len, want_lse=True, **kw)


@pytest.mark.parametrize("make", [prompt_call, decode_call])
def test_outputs_for_another_stream_are_not_memory_that_is_still_in_use(make):
    """A block that was freed while work of the current stream on it is still to come."""
    eng, shape, call = make(torch.Generator().manual_seed(213))
    want, want_lse = call()
    s = torch.cuda.Stream()
    for like in (want, want_lse):
        src, dst = torch.full_like(like, 3.0), torch.empty_like(like)
        torch.cuda.synchronize()
        busy()
        dst.copy_(src)
        del src
        out, lse = call(stream=s)
        torch.cuda.synchronize()
        assert (dst == 3).all() and torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("make", [prompt_call, decode_call])
def test_outputs_dropped_early_are_not_handed_on(make):
    """An output that is dropped while the stream it is written on has not come to it yet."""
    eng, shape, call = make(torch.Generator().manual_seed(214))
    call()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy(s)
    out, lse = call(stream=s)
    shapes = [(x.shape, x.dtype) for x in (out, lse)]
    del out, lse
    others = [torch.full(shape, 7.0, dtype=dtype, device="cuda") for shape, dtype in shapes for _ in range(2)]
    torch.cuda.synchronize()
    assert all((x == 7).all() for x in others)


@pytest.mark.parametrize("make", [prompt_call, decode_call])
def test_outputs_read_on_the_current_stream_and_dropped(make):
    """The other way round: the call's stream is ahead, the current one still reads the output."""
    eng, shape, call = make(torch.Generator().manual_seed(215))
    want, want_lse = call()
    s = torch.cuda.Stream()
    out, lse = call(stream=s)
    got = [torch.empty_like(out), torch.empty_like(lse)]
    s.synchronize()
    busy()
    got[0].copy_(out), got[1].copy_(lse)
    shapes = [(x.shape, x.dtype) for x in (out, lse)]
    del out, lse
    with torch.cuda.stream(s):
        others = [torch.full(shape, 7.0, dtype=dtype, device="cuda") for shape, dtype in shapes for _ in range(2)]
    torch.cuda.synchronize()
    assert torch.equal(got[0], want) and torch.equal(got[1], want_lse) and all((x == 7).all() for x in others)


@pytest.mark.parametrize("by_argument", [True, False])
def test_workspace_of_a_dropped_object_is_not_handed_on(by_argument):
    eng, shape, call = decode_call(torch.Generator().manual_seed(216))
    out, lse = call()
    n, s = binding.adaspark_attn_text_workspace_bytes(eng.handle), torch.cuda.Stream()
    torch.cuda.synchronize()
    busy(s)
    if by_argument:
        call(stream=s, out=out, lse=lse)
    else:
        with torch.cuda.stream(s):
            call(out=out, lse=lse)
    del eng, call
    gc.collect()
    others = [torch.full((n,), 9, dtype=torch.uint8, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert all((x == 9).all() for x in others)


def test_first_call_where_the_argument_is_a_stream_in_capture_is_refused():
    eng, shape, call = prompt_call(torch.Generator().manual_seed(217))
    want, _ = call()
    fresh, _, fresh_call = prompt_call(torch.Generator().manual_seed(217))
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g):
        s.wait_stream(torch.cuda.current_stream())
        with pytest.raises(binding.AdasparkError):
            fresh_call(stream=s)
        out, lse = call(stream=s)                                    # beside the capture's own stream
        torch.cuda.current_stream().wait_stream(s)
    for _ in range(3):
        out.zero_()
        g.replay()
        assert torch.equal(out, want)
