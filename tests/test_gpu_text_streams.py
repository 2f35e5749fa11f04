"""GPU tests of the text calls on a stream that is not torch's current one: what they report."""
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
