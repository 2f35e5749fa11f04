"""GPU tests of the text operators at the ends of what keys, queries and scores can hold, against plain forms in 64 bits."""
import math

import pytest
import torch

import text_util as tu
from paper_2604_08077_b200 import binding

pytestmark = pytest.mark.gpu


def draw(g, *shape, size=1.0):
    return (torch.randn(*shape, generator=g) * size).to(torch.bfloat16).cuda()


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def zero_cache(n_pages, Hkv, page, D, e4m3):
    dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    pages = [torch.zeros(n_pages, Hkv, page, D, dtype=dtype, device="cuda") for _ in range(2)]
    return binding.PagedCache(*pages, *([torch.zeros(n_pages, Hkv, page, dtype=torch.uint8, device="cuda") for _ in range(2)] if e4m3 else []))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (11, 1)])
@pytest.mark.parametrize("n", [5, 300, 6000])
def test_decode_rows_whose_scores_are_all_minus_infinity(e4m3, Hq, Hkv, n):
    """They give zeros, as rows without a key do; the other sequence of the call keeps its own."""
    g = torch.Generator().manual_seed(220)
    D, page = 128, 64
    per = -(-n // page)
    cache, eng = zero_cache(2 * per, Hkv, page, D, e4m3), tu.engine(Hq, Hkv, D)
    table, kv_len = torch.arange(2 * per, dtype=torch.int32, device="cuda").view(2, per), ints(n, n)
    k, v, q = draw(g, 2 * n, Hkv, D), draw(g, 2 * n, Hkv, D), draw(g, 2, Hq, D)
    k[n:] = 0
    k[n:, :, 0], q[1, :, 0] = (-2.0 ** 100, 2.0 ** 120) if e4m3 else (-math.inf, 1.0)     # (8 bits hold no infinity: a product beyond the range)
    eng.paged_write(cache, k, v, tu.cumulative([n, n]), table, kv_len)
    out, lse = eng.paged_decode(q, None, None, cache, table, kv_len, want_lse=True)
    assert eng.text_status() == 0
    assert (lse[1] == -math.inf).all() and (out[1] == 0).all()
    kk, vv = tu.sequence_values(cache, table, 0, n)
    want, wl, tol, ltol = tu.attend(q[:1], kk, vv, torch.tensor([n - 1], device="cuda"), D ** -0.5)
    tu.assert_close(out[:1], want, tol, "out")
    tu.assert_lse(lse[:1], wl, ltol)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,total", [(700, 700), (40, 9000)])
@pytest.mark.parametrize("level", [-3000.0, -30000.0, 0.0, 3000.0])
def test_prompt_whose_first_scores_are_all_minus_infinity(D, new, total, level):
    """The first 128 keys of every row (and some others) score minus infinity, those behind them far from zero: rows that see only the
    former give zeros, the others what the rest of their keys gives."""
    Hq, Hkv, g = 6, 2, torch.Generator().manual_seed(221)
    q, k, v = draw(g, new, Hq, D), draw(g, total, Hkv, D), draw(g, total, Hkv, D)
    k[:, :, :2], q[:, :, :2] = 0.0, 1.0
    k[128:, :, 1] = level
    hidden = torch.zeros(total, dtype=torch.bool, device="cuda")
    hidden[:128] = True
    hidden[200:270] = True
    k[hidden, :, 0] = -math.inf
    out, lse = tu.engine(Hq, Hkv, D).prompt(q, k, v, tu.cumulative([new]), tu.cumulative([total]), want_lse=True)
    last = torch.arange(new, device="cuda") + total - new
    seen = (~hidden).cumsum(0)[last] - 1                             # the last of the keys that are left
    want, wl, tol, ltol = tu.attend(q, k[~hidden], v[~hidden], seen, D ** -0.5)
    tu.assert_close(out, want, tol, "out")
    tu.assert_lse(lse, wl, ltol)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq", [7, 16])
@pytest.mark.parametrize("byte", [0, 1, 6, 20])
def test_decode_of_the_smallest_keys(D, Hq, byte):
    """Keys at the small end of what 8-bit pages hold (s = 0 is a power of two as any other), against queries as far at the large one:
    ordinary scores."""
    g = torch.Generator().manual_seed(222)
    page, n = 16, 200
    per = -(-n // page)
    cache = zero_cache(per, 1, page, D, True)
    cache.k_pages.copy_((torch.randn(per, 1, page, D, generator=g) * 32).cuda().to(torch.float8_e4m3fn))
    cache.v_pages.copy_((torch.randn(per, 1, page, D, generator=g) * 100).cuda().to(torch.float8_e4m3fn))
    cache.k_scale.fill_(byte)
    cache.v_scale.fill_(120)
    table = torch.arange(per, dtype=torch.int32, device="cuda").view(1, per)
    q = (torch.randn(1, Hq, D, generator=g).clamp(-3, 3) * 2.0 ** (122 - byte)).to(torch.bfloat16).cuda()
    out, lse = tu.engine(Hq, 1, D).paged_decode(q, None, None, cache, table, ints(n), want_lse=True)
    kk, vv = tu.sequence_values(cache, table, 0, n)
    want, wl, tol, ltol = tu.attend(q, kk, vv, torch.tensor([n - 1], device="cuda"), D ** -0.5)
    assert (wl - math.log(n)).abs().max() > 0.1                      # (the scores are not all zero)
    tu.assert_close(out, want, tol, "out")
    tu.assert_lse(lse, wl, ltol)


@pytest.mark.parametrize("D", [64, 128])
def test_decode_of_zero_keys_and_queries_beside_the_largest(D):
    """A score of zero is one whatever the powers of two around it."""
    cache, table, n = zero_cache(1, 1, 16, D, True), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), 9
    cache.k_pages[:, :, :, 0] = 256.0
    cache.v_pages.fill_(1.0)
    cache.k_scale.fill_(247)
    cache.v_scale.fill_(127)
    q = torch.zeros(1, 3, D, dtype=torch.bfloat16, device="cuda")
    q[0, 1:, 1] = 2.0 ** 127                                         # head 0: zeros; the others: at right angles to the keys
    q[0, 2, 2] = 2.0 ** -100
    out, lse = tu.engine(3, 1, D).paged_decode(q, None, None, cache, table, ints(n), want_lse=True)
    assert (out == 1).all()
    assert (lse - math.log(n)).abs().max() <= 2.0 ** -20


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n", [40, 300, 6000])
def test_decode_keys_that_are_no_numbers_show_in_the_logarithm(e4m3, n):
    """A whole first stretch of keys that are no numbers, ordinary ones behind them: neither the outputs nor the sum is a number."""
    g = torch.Generator().manual_seed(223)
    Hq, Hkv, D, page = 8, 2, 128, 16
    per = -(-n // page)
    cache, eng = zero_cache(per, Hkv, page, D, e4m3), tu.engine(Hq, Hkv, D)
    table, kv_len = torch.arange(per, dtype=torch.int32, device="cuda").view(1, per), ints(n)
    k, v, q = draw(g, n, Hkv, D), draw(g, n, Hkv, D), draw(g, 1, Hq, D)
    k[:32, 0, 5] = math.nan                                          # (all that a warp has of the first tile)
    eng.paged_write(cache, k, v, tu.cumulative([n]), table, kv_len)
    out, lse = eng.paged_decode(q, None, None, cache, table, kv_len, want_lse=True)
    assert torch.isnan(out[0, :4]).all() and torch.isnan(lse[0, :4]).all()
    kk, vv = tu.sequence_values(cache, table, 0, n)
    want, wl, tol, ltol = tu.attend(q[:, 4:], kk[:, 1:], vv[:, 1:], torch.tensor([n - 1], device="cuda"), D ** -0.5)
    tu.assert_close(out[:, 4:], want, tol, "out")
    tu.assert_lse(lse[:, 4:], wl, ltol)


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_appends_where_only_an_earlier_page_is_missing(e4m3):
    """The new token is written wherever its own place is there, whether the page that is not there lies in the same tile or in another."""
    g = torch.Generator().manual_seed(224)
    Hq, Hkv, D, page = 4, 2, 64, 16
    cache, eng = zero_cache(64, Hkv, page, D, e4m3), tu.engine(Hq, Hkv, D)
    table = torch.arange(60, dtype=torch.int32, device="cuda").view(3, 20)
    lens = [40, 300, 40]
    table[0, 0], table[1, 0], table[2, 2] = -1, 64, 64               # the tile of the new token | another tile | the new token's own page
    k, v, q = draw(g, 3, Hkv, D), draw(g, 3, Hkv, D), draw(g, 3, Hq, D)
    before = [x.clone() for x in tu.page_values(cache)]
    out, lse = eng.paged_decode(q, k, v, cache, table, ints(*lens), want_lse=True)
    assert eng.text_status() == 1
    assert (out == 0).all() and (lse == -math.inf).all()
    for was, now, x in zip(before, tu.page_values(cache), (k, v)):
        for b in (0, 1):
            pg, pl = int(table[b, (lens[b] - 1) // page]), (lens[b] - 1) % page
            assert torch.equal(now[pg, :, pl], tu.quantise(x[b])[0] if e4m3 else x[b].double())
            was[pg, :, pl] = now[pg, :, pl]
        assert torch.equal(was, now)


# (first, k0, k1) of a head, each a pair of bf16 numbers whose sum is the score: the largest of the first 128 keys, and one key in
# each half of the second 128, just below and above 2^100 times its weight.  Chosen so that a second rounding of the one's weight shows.
BOTH_HALVES = [
    (7.65625, -0.003936767578125, 77.0, -0.05859375, 77.0, -0.003814697265625), (18.0, 0.04150390625, 87.5, -0.1533203125, 87.5, -0.12890625),
    (2.125, -0.0023956298828125, 71.5, -0.08837890625, 71.5, -0.056640625), (8.375, -0.02587890625, 77.5, 0.150390625, 77.5, 0.1669921875),
    (18.75, 0.0274658203125, 88.0, 0.0625, 88.0, 0.09375), (26.375, 0.0302734375, 95.5, 0.1982421875, 95.5, 0.2333984375),
    (33.25, 0.07666015625, 102.5, 0.095703125, 102.5, 0.1572265625), (36.75, 0.001983642578125, 106.0, 0.056884765625, 106.0, 0.09375),
    (34.75, -0.06494140625, 104.0, -0.0257568359375, 104.0, 0.04345703125), (7.6875, -0.006927490234375, 77.0, -0.054931640625, 77.0, 0.01129150390625),
    (36.75, 0.0966796875, 106.0, 0.10302734375, 106.0, 0.166015625), (18.75, 0.0311279296875, 88.0, 0.06591796875, 88.0, 0.1015625),
    (22.25, -0.01348876953125, 91.5, 0.0010223388671875, 91.5, 0.095703125), (39.5, 0.0830078125, 109.0, -0.1279296875, 109.0, -0.09716796875),
    (18.75, 0.0150146484375, 88.0, 0.0703125, 88.0, 0.08642578125), (28.5, -0.00494384765625, 98.0, -0.2001953125, 98.0, -0.1728515625)]


def test_prompt_weights_are_rounded_once_when_both_halves_move_the_reference():
    """Scores of two exact products each, so that only these errors are left: 2^-22 of the score (its scale, its reference), 2^-17 for
    the exponential, both twice (numerator and sum), 2^-8 of a weight where it is rounded for the product with V, 2^-8 of the output."""
    H, D, n = len(BOTH_HALVES), 64, 256
    pairs = torch.tensor(BOTH_HALVES, dtype=torch.float64, device="cuda")
    q, k, v = (torch.zeros(r, H, D, dtype=torch.bfloat16, device="cuda") for r in (1, n, n))
    q[..., :2] = 1.0
    for at, (x, value) in {60: (0, 0.0), 150: (2, 1.0), 230: (4, -1.0)}.items():
        k[at, :, :2] = pairs[:, x:x + 2].to(torch.bfloat16)
        v[at] = value
    assert torch.equal(k[230, :, :2].double(), pairs[:, 4:])
    out, _ = tu.engine(H, H, D, softmax_scale=1.0).prompt(q, k, v, tu.cumulative([1]), tu.cumulative([n]))
    logits = k[..., :2].double().sum(-1)
    w = torch.softmax(logits, 0)
    want = (w[150] - w[230])[:, None]
    tol = 2.0 ** -8 * want.abs() + 2.0 ** -8 + 2 * (2.0 ** -22 * logits[230, :, None] + 2.0 ** -17)
    tu.assert_close(out[0], want.expand(H, D), tol.expand(H, D), "out")
