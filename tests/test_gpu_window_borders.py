"""Chunks by windows shorter than their tiles, over tiles that begin among the first tokens: steps masked at their end in front of ones masked at the
window's lower border, against 64 bits."""
import math

import pytest
import torch

from test_gpu_paged_prompt import ints, pool, rand, run_and_check
from text_util import cumulative, engine

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,new,ctx,page,window,sinks", [
    (4, 4, 128, [300], [0], 16, 100, 128), (4, 4, 64, [300], [0], 64, 48, 128), (4, 4, 64, [300], [0], 32, 48, 200), (28, 4, 128, [300], [0], 128, 8, 128),
    (28, 4, 64, [170, 40], [0, 100], 16, 8, 128), (8, 8, 64, [700], [0], 256, 1, 300), (4, 4, 128, [500, 3, 260], [0, 1000, 120], 16, 60, 256),
    (16, 8, 128, [129], [127], 64, 30, 128), (2, 2, 64, [5000], [0], 64, 200, 2000)])
def test_windows_shorter_than_a_tile_among_the_first_tokens(Hq, Hkv, D, new, ctx, page, window, sinks, e4m3):
    g = torch.Generator().manual_seed(window + sinks)
    eng = engine(Hq, Hkv, D)
    kv_len = [a + b for a, b in zip(new, ctx)]
    table, cache = pool(g, kv_len, page, Hkv, D, e4m3)
    q = rand(g, sum(new) + 2, Hq, D)
    run_and_check(eng, cache, table, q, cumulative(new, first=1), kv_len, window, sinks)


@pytest.mark.parametrize("e4m3", [False, True])
def test_many_such_tiles(e4m3):
    """More tiles than are cut into runs: whole ones, dealt to the pairs of CTAs."""
    g = torch.Generator().manual_seed(9)
    eng = engine(8, 8, 64)
    new, ctx = [300] * 24, [0] * 24
    table, cache = pool(g, new, 32, 8, 64, e4m3)
    run_and_check(eng, cache, table, rand(g, sum(new), 8, 64), cumulative(new), new, 100, 128)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("at", [50, 130, 260])
def test_values_that_are_no_numbers_at_such_borders(at, e4m3):
    """One among the first tokens, seen by every later row; ones behind them, seen by the rows whose window holds them."""
    g = torch.Generator().manual_seed(11)
    Hq = Hkv = 4
    D, page, n, window, sinks = 128, 16, 300, 100, 128
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, [n], page, Hkv, D, e4m3)
    q = rand(g, n, Hq, D)
    want, _ = run_and_check(eng, cache, table, q, [0, n], [n], window, sinks)
    x = cache.v_pages.view(torch.uint8) if e4m3 else cache.v_pages
    x[int(table[0, at // page]), 1, at % page, 9] = 0xff if e4m3 else math.nan
    out, _ = eng.paged_prompt(q, cache, ints([0, n]), table, ints([n]), window=window, sinks=sinks)
    assert eng.text_status() == 0
    p = torch.arange(n, device="cuda")
    sees = (p >= at) & ((p < at + window) | (at < sinks))
    assert out[sees, 1, 9].isnan().all()
    out[sees, 1, 9] = want[sees, 1, 9]
    assert torch.equal(out, want)
