"""GPU tests of the video calls on a stream that is not torch's current one: the memory that they allocate, the header they leave."""
import gc

import pytest
import torch

from paper_2604_08077_b200 import inputs

import parity_util as pu

pytestmark = pytest.mark.gpu


def busy(stream=None):
    """About 0.1 s of nothing on a stream."""
    with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
        torch.cuda._sleep(200_000_000)


def make(kind):
    wl = inputs.make_prefill("streams", seed=98, B=2, T=16, H=8, W=8, cube=(4, 4, 4), n_text=21, Hq=8, Hkv=2, D=128, top_p=0.8, offset_std=1.5)
    eng = pu.make_engine(wl, n_text_max=wl.n_text + 1)
    q, k, v = wl.q.cuda(), wl.k.cuda(), wl.v.cuda()
    if kind == "forward":
        return eng, lambda **kw: eng.forward(q, k, v, wl.n_text, want_selection=True, **kw)
    if kind == "chunk":
        return eng, lambda **kw: eng.forward_chunk(q, k, v, 0, 16, wl.n_text, want_selection=True, **kw)
    eng.forward(None, k, v, wl.n_text)
    g = torch.Generator().manual_seed(99)
    new = [torch.randn(2, 1, h, 128, generator=g).to(torch.bfloat16).cuda() for h in (8, 2, 2)]
    tl = torch.full((2,), wl.n_text, dtype=torch.int32, device="cuda")
    return eng, lambda **kw: eng.decode(*new, tl, want_selection=True, **kw)


KINDS = ["forward", "chunk", "decode"]


@pytest.mark.parametrize("kind", KINDS)
def test_outputs_for_another_stream_are_not_memory_that_is_still_in_use(kind):
    eng, call = make(kind)
    want, s = call(), torch.cuda.Stream()
    for like in want:
        src, dst = torch.full_like(like, 3), torch.empty_like(like)
        torch.cuda.synchronize()
        busy()
        dst.copy_(src)
        del src
        got = call(stream=s)
        torch.cuda.synchronize()
        assert (dst == 3).all() and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("kind", KINDS)
def test_outputs_dropped_early_are_not_handed_on(kind):
    eng, call = make(kind)
    shapes = [(x.shape, x.dtype) for x in call()]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy(s)
    got = call(stream=s)
    del got
    others = [torch.full(shape, 7, dtype=dtype, device="cuda") for shape, dtype in shapes for _ in range(2)]
    torch.cuda.synchronize()
    assert all((x == 7).all() for x in others)


@pytest.mark.parametrize("by_argument", [True, False])
@pytest.mark.parametrize("kind", KINDS)
def test_buffers_of_a_dropped_object_are_not_handed_on(kind, by_argument):
    eng, call = make(kind)
    first, s = call(), torch.cuda.Stream()
    buffers = [(x.shape, x.dtype) for x in (eng.k_cube, eng.v_cube, eng.cube_keys, eng.workspace)]
    torch.cuda.synchronize()
    busy(s)
    if by_argument:
        got = call(stream=s, out=first[0])
    else:
        with torch.cuda.stream(s):
            got = call(out=first[0])
    del eng, call
    gc.collect()
    others = [torch.full(shape, 7, dtype=dtype, device="cuda") for shape, dtype in buffers for _ in range(2)]
    torch.cuda.synchronize()
    assert all((x == 7).all() for x in others) and got is not None


def test_header_waits_for_calls_on_other_streams():
    eng, call = make("forward")
    call()
    want = bytes(eng.header())
    eng.workspace[:64] = 255
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy(s)
    call(stream=s)
    assert bytes(eng.header()) == want
