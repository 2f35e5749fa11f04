"""Attention of several new tokens, or of one, over a paged cache, all of it or a window of it, against 64 bits."""
import math

import pytest
import torch

from paper_2604_08077_b200 import binding
from text_util import assert_close, assert_lse, cumulative, engine, prompt_reference, scattered, sequence_values
from window_util import attend_masked, chunk_reference, hidden_from

pytestmark = pytest.mark.gpu


def rand(g, *shape, scale=1.0):
    return (scale * torch.randn(*shape, generator=g)).to(torch.bfloat16).cuda()


def pool(g, lens, page, Hkv, D, e4m3):
    table, n_pages = scattered(g, [-(-n // page) for n in lens])
    k, v = rand(g, n_pages, Hkv, page, D), rand(g, n_pages, Hkv, page, D)
    if not e4m3:
        return table, binding.PagedCache(k, v)
    # codes that are numbers, powers of two around those of values near 1
    codes = [(torch.randint(0, 127, k.shape, generator=g, dtype=torch.uint8) + 128 * torch.randint(0, 2, k.shape, generator=g, dtype=torch.uint8)).cuda() for _ in range(2)]
    scales = [torch.randint(116, 120, k.shape[:3], generator=g, dtype=torch.uint8).cuda() for _ in range(2)]
    return table, binding.PagedCache(*(c.view(torch.float8_e4m3fn) for c in codes), *scales)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def run_and_check(eng, cache, table, q, cu, kv_len, window=0, sinks=0, status=0):
    n = q.shape[0]
    cu_t, lens = cu if torch.is_tensor(cu) else ints(cu), ints(kv_len)
    cu = cu_t.tolist()
    out, lse = torch.full_like(q, 7.0, memory_format=torch.contiguous_format), torch.full(q.shape[:2], 7.0, device="cuda")
    out, lse = out.contiguous(), lse.contiguous()
    eng.paged_prompt(q, cache, cu_t, table, lens, window=window, sinks=sinks, out=out, lse=lse)
    assert eng.text_status() == status
    scale = q.shape[-1] ** -0.5
    mine, *want = chunk_reference(q, cu, kv_len, lambda b, m: sequence_values(cache, table, b, m), window, sinks, scale)
    assert (out[~mine] == 7).all() and (lse[~mine] == 7).all(), "rows of no sequence"
    assert n == out.shape[0]
    assert_close(out[mine], want[0][mine], want[2][mine], "out")
    assert_lse(lse[mine], want[1][mine], want[3][mine])
    return out, lse


SHAPES = [
    # new tokens, tokens before them, page, window, sinks
    ([41], [503], 16, 0, 0), ([1], [0], 16, 0, 0), ([5, 4, 1], [1000, 2047, 0], 64, 0, 0), ([130, 0, 1, 300], [77, 40, 128, 0], 32, 0, 0),
    ([17, 1, 64], [300, 128, 1000], 16, 100, 4), ([200], [900], 128, 128, 0), ([40, 3], [2000, 700], 64, 1, 0), ([33, 70], [1000, 0], 256, 257, 130),
    ([77, 3], [1111, 333], 16, 200, 0), ([77, 3], [1111, 333], 32, 131, 40), ([77], [1111], 64, 100, 129), ([150], [1111], 128, 300, 4), ([256, 5], [0, 640], 16, 37, 1), ([9], [4000], 64, 4000, 16), ([9], [4000], 32, 5000, 5000), ([100], [1500], 16, 64, 700)]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new,ctx,page,window,sinks", SHAPES)
@pytest.mark.parametrize("Hq,Hkv,D", [(28, 4, 128), (16, 4, 64)])
def test_chunks(Hq, Hkv, D, new, ctx, page, window, sinks, e4m3):
    g = torch.Generator().manual_seed(sum(new) + page)
    eng = engine(Hq, Hkv, D)
    kv_len = [a + b for a, b in zip(new, ctx)]
    table, cache = pool(g, kv_len, page, Hkv, D, e4m3)
    q = rand(g, sum(new) + 3, Hq, D, scale=1.5)
    run_and_check(eng, cache, table, q, cumulative(new, first=1), kv_len, window, sinks)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 4, 64), (16, 1, 64), (8, 8, 128), (16, 1, 128), (9, 3, 128), (5, 1, 64), (13, 1, 128)])
def test_groups(Hq, Hkv, D, e4m3):
    g = torch.Generator().manual_seed(Hq)
    eng = engine(Hq, Hkv, D)
    new, ctx = [65, 2, 150], [200, 513, 0]
    kv_len = [a + b for a, b in zip(new, ctx)]
    table, cache = pool(g, kv_len, 32, Hkv, D, e4m3)
    q = rand(g, sum(new), Hq, D)
    run_and_check(eng, cache, table, q, cumulative(new), kv_len)
    run_and_check(eng, cache, table, q, cumulative(new), kv_len, 90, 33)


@pytest.mark.parametrize("e4m3", [False, True])
def test_strided_rows_and_pages_of_a_larger_pool(e4m3):
    g = torch.Generator().manual_seed(3)
    Hq, Hkv, D, page = 8, 2, 128, 16
    eng = engine(Hq, Hkv, D)
    table, big = pool(g, [700, 90], page, Hkv, D, e4m3)
    parts = []
    for t in (big.k_pages, big.v_pages, big.k_scale, big.v_scale):
        if t is None:
            parts.append(None)
            continue
        apart = torch.zeros(2 * t.shape[0], *t.shape[1:], dtype=torch.uint8 if e4m3 else t.dtype, device="cuda")
        apart[::2] = t.view(torch.uint8) if e4m3 else t
        parts.append(apart.view(t.dtype)[::2])
    cache = binding.PagedCache(*parts)
    assert cache.page_stride == 2 * big.page_stride
    fused = rand(g, 60, Hq + 2 * Hkv, D)
    cu, lens = ints([0, 50, 60]), [700, 90]
    a = run_and_check(eng, cache, table, fused[:, :Hq], cu, lens, 50, 3)
    b = run_and_check(eng, big, table, fused[:, :Hq].contiguous(), cu, lens, 50, 3)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_long_caches_and_many_sequences(D, e4m3):
    g = torch.Generator().manual_seed(4)
    Hq, Hkv = 8, 2
    eng = engine(Hq, Hkv, D)
    kv_len = [30011, 9]
    table, cache = pool(g, kv_len, 64, Hkv, D, e4m3)
    q = rand(g, 24, Hq, D)
    run_and_check(eng, cache, table, q, [0, 20, 24], kv_len)
    run_and_check(eng, cache, table, q, [0, 20, 24], kv_len, 20000, 100)
    lens = [int(x) for x in torch.randint(1, 400, (70,), generator=g)]
    new = [min(n, int(x)) for n, x in zip(lens, torch.randint(0, 40, (70,), generator=g))]
    table, cache = pool(g, lens, 16, Hkv, D, e4m3)
    q = rand(g, sum(new), Hq, D)
    run_and_check(eng, cache, table, q, cumulative(new), lens)
    run_and_check(eng, cache, table, q, cumulative(new), lens, 50, 7)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 9)])
def test_what_is_hidden_may_be_anything(D, window, sinks, e4m3):
    """Places behind the last token, behind a row's own, between the first tokens and the window: no numbers there, and pages that are none."""
    g = torch.Generator().manual_seed(6)
    Hq, Hkv, page, n, r = 8, 2, 32, 1000, 21
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, [n], page, Hkv, D, e4m3)
    q = rand(g, r, Hq, D)
    want = run_and_check(eng, cache, table, q, [0, r], [n], window, sinks)
    k, v = (x.view(torch.uint8) if e4m3 else x for x in (cache.k_pages, cache.v_pages))
    odd = 0x7f if e4m3 else math.nan
    lo = max(n - r + 1 - window, 0) if window else 0
    for pos in list(range(n, -(-n // page) * page)) + list(range(sinks, lo)):
        for x in (k, v):
            x[int(table[0, pos // page]), :, pos % page] = odd
    other = torch.ones(cache.n_pages, dtype=torch.bool)
    other[table[0].long().cpu()] = False
    for x in (k, v):
        x[other.cuda()] = odd                                    # pages of no sequence
    def again():
        out, lse = eng.paged_prompt(q, cache, ints([0, r]), table, ints([n]), window=window, sinks=sinks, want_lse=True)
        assert eng.text_status() == 0
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    again()
    if window:
        for c in range(-(-sinks // page), lo // page):
            table[0, c] = [-1, cache.n_pages, 2 ** 31 - 1, -2 ** 31][c % 4]
        again()
    # a value that is no number, seen by the rows from its own on alone
    last = n - 5
    v[int(table[0, last // page]), 0, last % page, 3] = odd
    out, _ = eng.paged_prompt(q, cache, ints([0, r]), table, ints([n]), window=window, sinks=sinks)
    first = last - (n - r)
    assert torch.equal(out[:first], want[0][:first]) and torch.equal(out[first:, Hq // Hkv:], want[0][first:, Hq // Hkv:])
    assert out[first:, :Hq // Hkv, 3].isnan().all()
    rest = torch.arange(D, device="cuda") != 3
    assert torch.equal(out[first:, :Hq // Hkv][..., rest], want[0][first:, :Hq // Hkv][..., rest])


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_value_that_leaves_the_window(e4m3):
    """No number in the window of the first rows alone: the later ones do not see it."""
    g = torch.Generator().manual_seed(16)
    Hq, Hkv, D, page, n, r, window = 8, 2, 128, 16, 700, 64, 100
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, [n], page, Hkv, D, e4m3)
    q = rand(g, r, Hq, D)
    want, _ = run_and_check(eng, cache, table, q, [0, r], [n], window, 2)
    at = n - r + 1 - window + 20                                 # seen by the first 21 rows
    x = cache.v_pages.view(torch.uint8) if e4m3 else cache.v_pages
    x[int(table[0, at // page]), 1, at % page, 9] = 0xff if e4m3 else math.inf
    out, _ = eng.paged_prompt(q, cache, ints([0, r]), table, ints([n]), window=window, sinks=2)
    assert not torch.isfinite(out[:21, 4:, 9]).any()
    out[:21, 4:, 9] = want[:21, 4:, 9]
    assert torch.equal(out, want)


@pytest.mark.parametrize("e4m3", [False, True])
def test_scores_that_grow(e4m3):
    """Scores far apart, growing along the keys, so that a row's reference moves by more than weights can hold."""
    g = torch.Generator().manual_seed(7)
    Hq, Hkv, D, page, n, r = 8, 2, 128, 64, 1500, 30
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, [n], page, Hkv, D, e4m3)
    grow = torch.arange(n).float() / n
    for b, pos in enumerate(range(n)):
        where = (int(table[0, pos // page]), slice(None), pos % page)
        if e4m3:
            cache.k_scale[where] = 112 + int(14 * grow[b])
        else:
            cache.k_pages[where] = (cache.k_pages[where].float() * (0.1 + 60 * grow[b] ** 4)).to(torch.bfloat16)
    q = rand(g, r, Hq, D, scale=2.0)
    run_and_check(eng, cache, table, q, [0, r], [n])
    run_and_check(eng, cache, table, q, [0, r], [n], 800, 64)


@pytest.mark.parametrize("e4m3", [False, True])
def test_lengths_bounds_and_pages_out_of_range(e4m3):
    g = torch.Generator().manual_seed(8)
    Hq, Hkv, D, page = 4, 2, 64, 16
    eng = engine(Hq, Hkv, D)
    lens = [50, 60, 64, 40]
    table, cache = pool(g, lens, page, Hkv, D, e4m3)
    q = rand(g, 20, Hq, D)
    # kv_len below the new tokens, above the table, negative, in order
    kv_len = [3, 65, -4, 40]
    out, lse = torch.full((20, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((20, Hq), 7.0, device="cuda")
    eng.paged_prompt(q, cache, ints([0, 5, 10, 15, 20]), table, ints(kv_len), out=out, lse=lse)
    assert eng.text_status() == 1
    nothing = [0, 1] + list(range(5, 15))
    assert (out[nothing] == 0).all() and (lse[nothing] == -math.inf).all()
    for rows, b, n in ((slice(2, 5), 0, 3), (slice(15, 20), 3, 40)):
        k, v = sequence_values(cache, table, b, n)
        r = rows.stop - rows.start
        want, wl, tol, ltol = attend_masked(q[rows], k, v, hidden_from(n - r, r, n, 0, 0), D ** -0.5)
        assert_close(out[rows], want, tol, "out")
        assert_lse(lse[rows], wl, ltol)
    # bounds that leave the tensors or decrease: those sequences are left out
    out.fill_(7.0)
    eng.paged_prompt(q, cache, ints([0, 5, 30, 15, 20]), table, ints(lens), out=out, lse=lse)
    assert eng.text_status() == 1
    assert (out[5:15] == 7).all()
    for rows, b, n in ((slice(0, 5), 0, 50), (slice(15, 20), 3, 40)):
        k, v = sequence_values(cache, table, b, n)
        want, _, tol, _ = attend_masked(q[rows], k, v, hidden_from(n - 5, 5, n, 0, 0), D ** -0.5)
        assert_close(out[rows], want, tol, "out")
    # a page that is not there counts as zeros
    table[1, 2] = cache.n_pages + 5
    k, v = sequence_values(cache, torch.where(table == cache.n_pages + 5, 0, table), 1, 60)
    k[32:48], v[32:48] = 0, 0
    out, lse = eng.paged_prompt(q, cache, ints([0, 0, 20, 20, 20]), table, ints([0, 60, 0, 0]), want_lse=True)
    assert eng.text_status() == 1
    want, wl, tol, ltol = attend_masked(q, k, v, hidden_from(40, 20, 60, 0, 0), D ** -0.5)
    assert_close(out, want, tol, "out")
    assert_lse(lse, wl, ltol)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 64), (28, 4, 128)])
def test_rows_in_front_of_the_first_token_with_a_window_of_any_length(Hq, Hkv, D, e4m3):
    g = torch.Generator().manual_seed(80)
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, [144], 16, Hkv, D, e4m3)
    q = rand(g, 90, Hq, D)
    out, lse = eng.paged_prompt(q, cache, ints([0, 90]), table, ints([60]), window=2 ** 31 - 1, sinks=5, want_lse=True)
    assert eng.text_status() == 1
    assert (out[:30] == 0).all() and (lse[:30] == -math.inf).all()
    k, v = sequence_values(cache, table, 0, 60)
    want, wl, tol, ltol = attend_masked(q[30:], k, v, hidden_from(0, 60, 60, 0, 0), D ** -0.5)
    assert_close(out[30:], want, tol, "out")
    assert_lse(lse[30:], wl, ltol)


def test_empty_calls():
    eng = engine(4, 2, 64)
    cache = eng.paged_cache(2, 16)
    table = torch.zeros(3, 1, dtype=torch.int32, device="cuda")
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = eng.paged_prompt(q, cache, ints([0, 0, 0, 0]), table, ints([0, 1, 0]), want_lse=True)
    assert out.shape == q.shape and lse.shape == (0, 4)
    q = torch.zeros(6, 4, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7)
    eng.paged_prompt(q, cache, ints([3, 3, 3, 3]), table, ints([0, 1, 0]), out=out)
    assert (out == 7).all() and eng.text_status() == 0


def test_as_prompt_over_what_is_read_back():
    g = torch.Generator().manual_seed(10)
    Hq, Hkv, D, page = 28, 4, 128, 64
    eng = engine(Hq, Hkv, D)
    new, kv_len = [100, 3], [1100, 515]
    table, cache = pool(g, kv_len, page, Hkv, D, True)
    q = rand(g, 103, Hq, D)
    cu, all_ = cumulative(new), cumulative(kv_len)
    out, lse = eng.paged_prompt(q, cache, cu, table, ints(kv_len), want_lse=True)
    k, v = torch.empty(sum(kv_len), Hkv, D, dtype=torch.bfloat16, device="cuda"), torch.empty(sum(kv_len), Hkv, D, dtype=torch.bfloat16, device="cuda")
    eng.paged_read(cache, all_, table, ints(kv_len), k, v)
    out2, lse2 = eng.prompt(q, k, v, cu, all_, want_lse=True)
    _, _, _, tol, ltol = prompt_reference(q, k, v, cu, all_, D ** -0.5)
    assert_close(out, out2.double(), 2 * tol, "out")
    assert_lse(lse, lse2.double(), 2 * ltol)


def test_a_captured_step_with_new_lengths():
    """Append, chunk and decode in one graph, replayed with other tokens, lengths and pages; two objects of their own side by side."""
    g = torch.Generator().manual_seed(12)
    Hq, Hkv, D, page = 8, 2, 64, 16
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, [400, 300], page, Hkv, D, False)
    rotary = binding.Rotary(D)
    q, k, v = rand(g, 12, Hq, D), rand(g, 12, Hkv, D), rand(g, 12, Hkv, D)
    cu, lens = ints([0, 9, 12]), ints([100, 80])

    def step():
        qo = eng.paged_append(cache, q, k, v, cu, table, lens, rotary)
        return eng.paged_prompt(qo, cache, cu, table, lens, window=70, sinks=3, want_lse=True)
    step()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out, lse = step()
    torch.cuda.synchronize()
    for kv in ([100, 80], [399, 3], [12, 250]):
        lens.copy_(ints(kv))
        for x in (q, k, v):
            x.copy_(rand(g, *x.shape))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        want = step()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert eng.text_status() == 0


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 31 - 1), (2 ** 30, 2 ** 30)])
def test_windows_that_hide_nothing(window, sinks, e4m3):
    g = torch.Generator().manual_seed(141)
    Hq, Hkv, D, page = 8, 2, 128, 32
    eng = engine(Hq, Hkv, D)
    new, kv_len = [3, 40, 0, 1], [3, 1700, 0, 900]
    table, cache = pool(g, kv_len, page, Hkv, D, e4m3)
    q, cu = rand(g, 44, Hq, D), cumulative(new)
    run_and_check(eng, cache, table, q, cu, kv_len, window, sinks)
    got = eng.paged_decode(q[:4], None, None, cache, table, ints(kv_len), window=window, sinks=sinks, want_lse=True)
    want = eng.paged_decode(q[:4], None, None, cache, table, ints(kv_len), want_lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert eng.text_status() == 0


def test_two_captured_steps_in_turn():
    """Graphs of one object, replayed one behind the other in any order: they share its workspace."""
    g = torch.Generator().manual_seed(142)
    Hq, Hkv, D, page = 28, 4, 128, 64
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, [9000, 5000], page, Hkv, D, True)
    cu, lens, rotary = ints([0, 4, 5]), ints([9000, 5000]), binding.Rotary(D)
    q, k, v, pos = rand(g, 5, Hq, D), rand(g, 5, Hkv, D), rand(g, 5, Hkv, D), ints([1, 2, 3, 4, 5])

    def chunk():
        return eng.paged_prompt(eng.rotate(q, None, pos, rotary)[0], cache, cu, table, lens)[0]

    def token():
        return eng.paged_decode(q[:2], k[:2], v[:2], cache, table, lens, window=4000, sinks=4)[0]
    want = []
    graphs, outs = [], []
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        token()
        for f in (chunk, token):
            want.append(f().clone())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                outs.append(f())
            graphs.append(graph)
    torch.cuda.synchronize()
    for i in (0, 1, 1, 0, 0, 1):
        outs[i].fill_(7.0)
        graphs[i].replay()
        graphs[1 - i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_another_stream():
    g = torch.Generator().manual_seed(14)
    Hq, Hkv, D, page, n = 8, 2, 128, 32, 3000
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, [n], page, Hkv, D, True)
    q = rand(g, 50, Hq, D)
    want, _ = eng.paged_prompt(q, cache, ints([0, 50]), table, ints([n]))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    cu, lens = ints([0, 50]), ints([n])
    torch.cuda.synchronize()
    out, _ = eng.paged_prompt(q, cache, cu, table, lens, stream=s)
    s.synchronize()
    assert torch.equal(out, want)


# ---------------------------------------------------------------------------------------------------------------- one new token, by a window

@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 1), (100, 0), (128, 4), (257, 130), (1000, 70), (5000, 3), (64, 5000), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("Hq,Hkv,D,page", [(28, 4, 128, 16), (16, 4, 64, 64), (16, 1, 128, 256)])
def test_decode_window(Hq, Hkv, D, page, window, sinks, e4m3):
    g = torch.Generator().manual_seed(window % 1000)
    eng = engine(Hq, Hkv, D)
    kv_len = [700, 0, 1, 3001, 128, 129, 64, 1300]
    table, cache = pool(g, kv_len, page, Hkv, D, e4m3)
    q = rand(g, len(kv_len), Hq, D)
    append = rand(g, len(kv_len), Hkv, D) if window % 2 else None
    out, lse = eng.paged_decode(q, append, append, cache, table, ints(kv_len), window=window, sinks=sinks, want_lse=True)
    assert eng.text_status() == 0
    for b, n in enumerate(kv_len):
        if n == 0:
            assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
            continue
        k, v = sequence_values(cache, table, b, n)
        want, wl, tol, ltol = attend_masked(q[b:b + 1], k, v, hidden_from(n - 1, 1, n, window, sinks), D ** -0.5)
        assert_close(out[b:b + 1], want, tol, f"out {b}")
        assert_lse(lse[b:b + 1], wl, ltol)
    if window > 5000:
        plain, plse = eng.paged_decode(q, None, None, cache, table, ints(kv_len), want_lse=True)
        assert torch.equal(out, plain) and torch.equal(lse, plse)


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_window_over_pages_given_back(e4m3):
    g = torch.Generator().manual_seed(21)
    Hq, Hkv, D, page, window, sinks = 8, 2, 128, 16, 100, 20
    eng = engine(Hq, Hkv, D)
    kv_len = [5000, 333]
    table, cache = pool(g, kv_len, page, Hkv, D, e4m3)
    q = rand(g, 2, Hq, D)
    want = eng.paged_decode(q, None, None, cache, table, ints(kv_len), window=window, sinks=sinks, want_lse=True)
    for x in (cache.k_pages, cache.v_pages):
        x = x.view(torch.uint8) if e4m3 else x
        for b, n in enumerate(kv_len):
            for pos in list(range(sinks, n - window)) + list(range(n, -(-n // page) * page)):
                x[int(table[b, pos // page]), :, pos % page] = 0x7f if e4m3 else math.nan
    for b, n in enumerate(kv_len):
        table[b, -(-sinks // page):(n - window) // page] = -1
    got = eng.paged_decode(q, None, None, cache, table, ints(kv_len), window=window, sinks=sinks, want_lse=True)
    assert eng.text_status() == 0
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    table[1, 0] = -1                                             # of the first ones
    out, lse = eng.paged_decode(q, None, None, cache, table, ints(kv_len), window=window, sinks=sinks, want_lse=True)
    assert eng.text_status() == 1
    assert torch.equal(out[0], want[0][0]) and (out[1] == 0).all() and (lse[1] == -math.inf).all()


def test_decode_window_is_a_chunk_of_one():
    g = torch.Generator().manual_seed(22)
    Hq, Hkv, D, page = 28, 4, 128, 64
    eng = engine(Hq, Hkv, D)
    kv_len = [4000, 1, 200]
    table, cache = pool(g, kv_len, page, Hkv, D, False)
    q = rand(g, 3, Hq, D)
    out, lse = eng.paged_decode(q, None, None, cache, table, ints(kv_len), window=1500, sinks=4, want_lse=True)
    out2, lse2 = eng.paged_prompt(q, cache, ints([0, 1, 2, 3]), table, ints(kv_len), window=1500, sinks=4, want_lse=True)
    _, _, _, tol, ltol = chunk_reference(q, [0, 1, 2, 3], kv_len, lambda b, m: sequence_values(cache, table, b, m), 1500, 4, D ** -0.5)
    assert_close(out, out2.double(), 2 * tol, "out")
    assert_lse(lse, lse2.double(), 2 * ltol)


# ---------------------------------------------------------------------------------------------------------------- 8-bit pages as the tensor cores take them

def one_sequence(g, n, page, Hkv, D):
    table, cache = pool(g, [n], page, Hkv, D, True)
    return table, cache, sequence_values(cache, table, 0, n)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q_power,k_power", [(110, -105), (-105, 100), (60, -60), (0, 0)])
def test_powers_of_two_at_opposite_ends(D, q_power, k_power):
    """Queries and keys whose powers of two cancel: the scores are ordinary ones."""
    g = torch.Generator().manual_seed(30)
    Hq, Hkv, page, n, r = 8, 2, 16, 700, 20
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, [n], page, Hkv, D, True)
    cache.k_scale.copy_((cache.k_scale.to(torch.int32) + k_power).clamp(0, 247).to(torch.uint8))
    q = (0.02 * torch.randn(r, Hq, D, generator=g) * 2.0 ** q_power).to(torch.bfloat16).cuda()
    run_and_check(eng, cache, table, q, [0, r], [n])


def test_queries_with_large_elements():
    """One value of a row 2^12 times the others: those are held to 2^-18 of it, which moves a score by 2^-18 max|q| sum|k| at most, on top of
    what the bounds have."""
    g = torch.Generator().manual_seed(31)
    Hq, Hkv, D, page, n, r = 8, 2, 128, 64, 900, 30
    eng = engine(Hq, Hkv, D)
    table, cache, (k, v) = one_sequence(g, n, page, Hkv, D)
    q = rand(g, r, Hq, D)
    q[..., 17] *= 64
    q[::3, :, 17] *= 64
    for x in (cache.k_pages.view(torch.uint8),):
        x[..., 17] &= 0x87                                       # the keys are small where the queries are large
    k, v = sequence_values(cache, table, 0, n)
    out, lse = eng.paged_prompt(q, cache, ints([0, r]), table, ints([n]), want_lse=True)
    want, wl, tol, ltol = attend_masked(q, k, v, hidden_from(n - r, r, n, 0, 0), D ** -0.5)
    e = q.double().abs().amax(-1) * 2.0 ** -18 * k.abs().sum(-1).amax() * D ** -0.5
    size = v.abs().amax()
    assert_close(out, want, tol + (2 * e * size)[..., None], "out")
    assert_lse(lse, wl, ltol + e)


@pytest.mark.parametrize("D", [64, 128])
def test_every_code_with_every_power_of_two(D):
    """A token that sees itself alone gives its value back, whatever code and power of two it has."""
    eng = engine(1, 1, D)
    per = 256 // D if D < 256 else 1
    codes = torch.arange(256, dtype=torch.uint8).repeat(255).view(-1, D)
    s = torch.arange(255, dtype=torch.uint8).repeat_interleave(per)
    n = codes.shape[0]
    kp, vp = torch.zeros(n, 1, 16, D, dtype=torch.uint8, device="cuda"), torch.zeros(n, 1, 16, D, dtype=torch.uint8, device="cuda")
    vs = torch.full((n, 1, 16), 127, dtype=torch.uint8, device="cuda")
    vp[:, 0, 0], vs[:, 0, 0] = codes.cuda(), s.cuda()
    cache = binding.PagedCache(kp.view(torch.float8_e4m3fn), vp.view(torch.float8_e4m3fn), torch.full_like(vs, 127), vs)
    table, one, cu = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous(), ints([1] * n), torch.arange(n + 1, dtype=torch.int32, device="cuda")
    q = torch.ones(n, 1, D, dtype=torch.bfloat16, device="cuda")
    out, _ = eng.paged_prompt(q, cache, cu, table, one)
    want, k = torch.empty_like(out), torch.empty_like(out)
    eng.paged_read(cache, cu, table, one, k, want)
    assert eng.text_status() == 0
    assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.nan_to_num(), want.nan_to_num())


def test_keys_and_queries_that_are_no_numbers():
    g = torch.Generator().manual_seed(33)
    Hq, Hkv, D, page, n, r = 8, 2, 128, 16, 500, 40
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, [n], page, Hkv, D, True)
    q = rand(g, r, Hq, D)
    want, _ = run_and_check(eng, cache, table, q, [0, r], [n])
    at = n - 10                                                  # a key that the last ten rows see
    kept = cache.k_pages.view(torch.uint8)[int(table[0, at // page]), 1, at % page, 5].clone()
    cache.k_pages.view(torch.uint8)[int(table[0, at // page]), 1, at % page, 5] = 0x7f
    out, _ = eng.paged_prompt(q, cache, ints([0, r]), table, ints([n]))
    assert torch.equal(out[:r - 10], want[:r - 10]) and torch.equal(out[:, :4], want[:, :4]) and out[r - 10:, 4:].isnan().all()
    cache.k_pages.view(torch.uint8)[int(table[0, at // page]), 1, at % page, 5] = kept
    q[3, 2, 7], q[20, 5, 0] = math.nan, math.inf
    out, _ = eng.paged_prompt(q, cache, ints([0, r]), table, ints([n]))
    assert out[3, 2].isnan().all() and out[20, 5].isnan().all()
    out[3, 2], out[20, 5] = want[3, 2], want[20, 5]
    assert torch.equal(out, want)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (3000, 10)])
def test_runs_that_end_anywhere(window, sinks, e4m3):
    """Sequences that the pairs' runs cut at any place, one that is a run of many, ones without rows between them."""
    g = torch.Generator().manual_seed(34)
    Hq, Hkv, D, page = 16, 4, 64, 32
    eng = engine(Hq, Hkv, D)
    new, kv_len = [1, 0, 33, 5, 64, 130, 0, 7, 2], [9000, 500, 2000, 12345, 1600, 130, 0, 4100, 2]
    table, cache = pool(g, kv_len, page, Hkv, D, e4m3)
    q = rand(g, sum(new), Hq, D)
    first = run_and_check(eng, cache, table, q, cumulative(new), kv_len, window, sinks)
    again = run_and_check(eng, cache, table, q, cumulative(new), kv_len, window, sinks)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("e4m3", [False, True])
def test_many_long_tiles(e4m3):
    """More tiles than four a pair, dealt longest first: long ones alike, and ones of two lengths."""
    g = torch.Generator().manual_seed(35)
    Hq, Hkv, D, page = 16, 8, 64, 64
    eng = engine(Hq, Hkv, D)
    for new, kv_len in (([40] * 45, [13000] * 45), ([300, 129] * 10, [1800, 130] * 10)):
        order = torch.randperm(64 * -(-max(kv_len) // page) // 4, generator=g).to(torch.int32)
        width = -(-max(kv_len) // page)
        table = torch.stack([order[torch.randint(0, order.numel(), (width,), generator=g)] for _ in kv_len]).cuda()   # (sequences may share what nobody writes)
        k, v = rand(g, order.numel(), Hkv, page, D), rand(g, order.numel(), Hkv, page, D)
        if e4m3:
            k, v = (x.float().mul(16).to(torch.float8_e4m3fn) for x in (k, v))
            cache = binding.PagedCache(k, v, *(torch.full(k.shape[:3], 123, dtype=torch.uint8, device="cuda") for _ in range(2)))
        else:
            cache = binding.PagedCache(k, v)
        q = rand(g, sum(new), Hq, D)
        out, lse = eng.paged_prompt(q, cache, cumulative(new), table, ints(kv_len), want_lse=True)
        assert eng.text_status() == 0
        at = 0
        for b, (r, n) in enumerate(zip(new, kv_len)):
            rows, at = slice(at, at + r), at + r
            if b % 9:
                continue
            keys, values = sequence_values(cache, table, b, n)
            want, wl, tol, ltol = attend_masked(q[rows], keys, values, hidden_from(n - r, r, n, 0, 0), D ** -0.5)
            if e4m3:                                             # q in two parts: 2^-18 of its largest magnitude, as a score
                e = q[rows].double().abs().amax(-1) * 2.0 ** -18 * keys.abs().sum(-1).amax() * D ** -0.5
                tol, ltol = tol + (2 * e * values.abs().amax())[..., None], ltol + e
            assert_close(out[rows], want, tol, f"out {b}")
            assert_lse(lse[rows], wl, ltol)


def test_pages_far_apart():
    """A pool of more than 2^31 values: what lies at its end is written and read there."""
    g = torch.Generator().manual_seed(36)
    Hq, Hkv, D, page, n_pages = 8, 4, 128, 64, 70000
    eng = engine(Hq, Hkv, D)
    cache = binding.PagedCache(*(torch.empty(n_pages, Hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    assert cache.k_pages.numel() > 2 ** 31
    n, r = 500, 500
    table = (n_pages - 1 - torch.randperm(8, generator=g).to(torch.int32) * 100).cuda()[None].contiguous()
    q, k, v = rand(g, r, Hq, D), rand(g, r, Hkv, D), rand(g, r, Hkv, D)
    eng.paged_append(cache, None, k, v, ints([0, r]), table, ints([n]))
    at = torch.arange(n, device="cuda")
    assert torch.equal(cache.k_pages[table[0].long()[at // page], :, at % page], k) and torch.equal(cache.v_pages[table[0].long()[at // page], :, at % page], v)
    out, _ = eng.paged_prompt(q[-40:], cache, ints([0, 40]), table, ints([n]), window=300, sinks=3)
    want, _, tol, _ = attend_masked(q[-40:], k, v, hidden_from(n - 40, 40, n, 300, 3), D ** -0.5)
    assert_close(out, want, tol, "out")
    one, _ = eng.paged_decode(q[-1:], None, None, cache, table, ints([n]), window=300, sinks=3)
    assert_close(one, want[-1:], tol[-1:], "decode")
    assert eng.text_status() == 0


def test_refusals_of_the_binding():
    eng = engine(4, 2, 64)
    cache = eng.paged_cache(4, 16)
    other = engine(4, 4, 64).paged_cache(4, 16)
    q, k, table, lens, cu = torch.zeros(5, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="cuda"), ints([[0], [1]]), ints([5, 0]), ints([0, 5, 5])
    rope, wide = binding.Rotary(64, sections=[8, 8, 8]), binding.Rotary(128)
    pos = torch.zeros(3, 5, dtype=torch.int32, device="cuda")

    def refused(fn, *a, **kw):
        with pytest.raises(binding.AdasparkError) as e:
            fn(*a, **kw)
        return e.value.status == binding.ERR_INVALID_ARG
    assert refused(eng.paged_prompt, q, other, cu, table, lens) and refused(eng.paged_prompt, q.half(), cache, cu, table, lens)
    assert refused(eng.paged_prompt, k, cache, cu, table, lens) and refused(eng.paged_prompt, q, cache, cu[:2], table, lens)
    assert refused(eng.paged_prompt, q, cache, cu, table, lens, window=-1) and refused(eng.paged_prompt, q, cache, cu, table, lens, window=4, sinks=-2)
    assert refused(eng.paged_prompt, q, cache, cu, table.cpu(), lens) and refused(eng.paged_prompt, q, cache, cu, table, lens, out=q[:4])
    assert refused(eng.paged_prompt, q, cache, cu.long(), table, lens) and refused(eng.paged_prompt, q, cache, cu, table, lens, lse=torch.zeros(5, 4, dtype=torch.float64, device="cuda"))
    assert refused(eng.paged_decode, q[:2], None, None, cache, table, lens, window=-3) and refused(eng.paged_decode, q[:2], None, None, cache, table, lens, sinks=-1)
    assert refused(eng.rotate, q, k, pos, wide) and refused(eng.rotate, q, k, None, rope) and refused(eng.rotate, None, None)
    assert refused(eng.rotate, q, k, pos[:2], rope) and refused(eng.rotate, q, k, pos.long(), rope) and refused(eng.rotate, q, k[:4], pos, rope)
    assert refused(eng.rotate, q, k, pos.cpu(), rope) and refused(eng.rotate, q, None, pos, rope, k_out=k) and refused(eng.rotate, q, k, pos, rope, q_out=q[:3])
    assert refused(eng.rotate, q, k, q_norm=torch.zeros(128, dtype=torch.bfloat16, device="cuda")) and refused(eng.rotate, q, k, eps=-1.0)
    assert refused(eng.rotate, q.expand(5, 4, 64)[:, :1].expand(5, 4, 64), k)                # one row for all heads
    assert refused(eng.paged_append, cache, q, k, k[:4], cu, table, lens) and refused(eng.paged_append, cache, None, k, k, cu, table, lens, q_out=q)
    assert refused(eng.paged_append, cache, q, k, k, cu, table, lens, rope, positions=pos[0].contiguous())
    assert eng.text_status() == 0
