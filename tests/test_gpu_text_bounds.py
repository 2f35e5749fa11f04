"""GPU tests of the paged cache's calls with sequence bounds (cu) that leave the tensors or decrease: reported, and never followed."""
import pytest
import torch

import text_util as tu
from paper_2604_08077_b200 import binding

pytestmark = pytest.mark.gpu

N, HKV, D, PAGE = 64, 2, 64, 16
INT_MIN = -(1 << 31)


def make(e4m3):
    g = torch.Generator().manual_seed(200)
    shape = (12, HKV, PAGE, D)
    if e4m3:
        pages = [torch.randint(0, 120, shape, generator=g, dtype=torch.uint8).cuda().view(torch.float8_e4m3fn) for _ in range(2)]
        scales = [torch.randint(100, 140, shape[:3], generator=g, dtype=torch.uint8).cuda() for _ in range(2)]
    else:
        pages, scales = [torch.randn(shape, generator=g).to(torch.bfloat16).cuda() for _ in range(2)], [None, None]
    k, v = (torch.randn(N, HKV, D, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    return binding.PagedCache(*pages, *scales), k, v, torch.arange(12, dtype=torch.int32, device="cuda").view(2, 6)


def raw(cache):
    return [t.clone().view(torch.uint8) for t in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale) if t is not None]


# cu, kv_len, the rows that have a place and the sequence each is of, rows of a sequence that is left out
CASES = [
    ([0, 20, 65], [20, 45], {0: range(0, 20)}, range(20, 64)),       # one row more than the tensors hold
    ([-5, 20, 64], [25, 44], {1: range(20, 64)}, range(0, 20)),      # begins in front of them
    ([0, -3, 64], [20, 80], {}, range(0, 64)),                       # decreasing: no sequence has bounds
    ([0, 40, 20], [40, 20], {0: range(0, 20)}, []),                  # decreasing: rows 20 .. 39 lie behind the last bound
    ([0, 64, 70], [64, 6], {0: range(0, 64)}, []),                   # a whole sequence behind them
    ([0, 20, 64], [INT_MIN, 44], {1: range(20, 64)}, range(0, 20)),  # a length far out of range
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("cu,kv_len,there,left_out", CASES)
def test_bounds_out_of_range_are_reported_and_not_followed(e4m3, cu, kv_len, there, left_out):
    cache, k, v, table = make(e4m3)
    eng = tu.engine(2 * HKV, HKV, D)
    bounds, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (cu, kv_len))
    before = raw(cache)
    eng.paged_write(cache, k, v, bounds, table, lens)
    assert eng.text_status() == 1
    held = []
    for b, rows in there.items():
        for i in rows:
            pos = kv_len[b] - (cu[b + 1] - i)
            held.append((i, int(table[b, pos // PAGE]), pos % PAGE))
    row, page, place = (torch.tensor([h[x] for h in held], dtype=torch.long, device="cuda") for x in range(3))
    for x, values in zip((k, v), tu.page_values(cache)):
        assert torch.equal(values[page, :, place], tu.quantise(x[row])[0] if e4m3 else x[row].double())
    for was, now in zip(before, raw(cache)):
        now[page, :, place] = was[page, :, place]
        assert torch.equal(was, now)
    ko, vo = (torch.full((N, HKV, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    eng.paged_read(cache, bounds, table, lens, ko, vo)
    assert eng.text_status() == 1
    for got, values in zip((ko, vo), tu.page_values(cache)):
        assert torch.equal(got[row].double(), values[page, :, place])
        assert (got[torch.tensor(list(left_out), dtype=torch.long, device="cuda")] == 0).all()


def test_many_sequences_one_of_them_out_of_range():
    """The report does not depend on where in the batch the bad bound stands, nor on its sequence having a row in the tensors."""
    cache, k, v, _ = make(False)
    eng = tu.engine(2 * HKV, HKV, D)
    B = 700
    table, lens = torch.zeros(B, 1, dtype=torch.int32, device="cuda"), torch.ones(B, dtype=torch.int32, device="cuda")
    for at in (0, 31, 32, 255, 256, 699):
        cu = [1] * (B + 1)
        cu[at + 1:] = [N + 1] * (B - at)
        eng.paged_write(cache, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), table, lens)
        assert eng.text_status() == 1, at
    eng.paged_write(cache, k, v, torch.tensor([1] * B + [2], dtype=torch.int32, device="cuda"), table, lens)
    assert eng.text_status() == 0


@pytest.mark.parametrize("e4m3", [False, True])
def test_rows_with_the_same_place_leave_the_others_alone(e4m3):
    """Such a place holds a mixture; every other one what belongs there, and nothing else is written."""
    cache, k, v, _ = make(e4m3)
    eng = tu.engine(2 * HKV, HKV, D)
    table = torch.tensor([[3], [3], [5], [3], [7]], dtype=torch.int32, device="cuda")       # three sequences write to page 3
    cu, kv_len = tu.cumulative([1, 2, 10, 4, 16]), torch.tensor([4, 4, 10, 4, 16], dtype=torch.int32, device="cuda")
    before = raw(cache)
    eng.paged_write(cache, k, v, cu, table, kv_len)
    assert eng.text_status() == 0
    held = [(i, int(table[b, 0]), int(kv_len[b]) - (int(cu[b + 1]) - i)) for b in (2, 4) for i in range(int(cu[b]), int(cu[b + 1]))]
    held += [(13, 3, 0), (14, 3, 1)]                                     # (the fourth sequence's first two rows have places of their own)
    row, page, place = (torch.tensor([h[x] for h in held], dtype=torch.long, device="cuda") for x in range(3))
    for x, values in zip((k, v), tu.page_values(cache)):
        assert torch.equal(values[page, :, place], tu.quantise(x[row])[0] if e4m3 else x[row].double())
    for was, now in zip(before, raw(cache)):
        now[page, :, place] = was[page, :, place]
        now[3, :, 2:4] = was[3, :, 2:4]
        assert torch.equal(was, now)
