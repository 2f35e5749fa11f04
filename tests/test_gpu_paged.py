"""GPU tests of the paged cache (written, quantised, read back) and of the decode step over its pages, against plain forms in 64 bits."""
import math

import pytest
import torch

import text_util as tu
from paper_2604_08077_b200 import binding

pytestmark = pytest.mark.gpu


def draw(g, *shape, size=1.0):
    return (torch.randn(*shape, generator=g) * size).to(torch.bfloat16).cuda()


def make_cache(g, n_pages, Hkv, page, D, e4m3, interleaved=False):
    """A cache whose pages already hold something (of any kind): what a call does not write has to stay."""
    if e4m3:
        pages = [torch.randint(0, 255, (n_pages, Hkv, page, D), generator=g, dtype=torch.uint8).cuda().view(torch.float8_e4m3fn) for _ in range(2)]
        scales = [torch.randint(0, 255, (n_pages, Hkv, page), generator=g, dtype=torch.uint8).cuda() for _ in range(2)]
    else:
        pages, scales = [draw(g, n_pages, Hkv, page, D) for _ in range(2)], [None, None]
    if interleaved:
        both = torch.stack([p.view(torch.uint8) for p in pages], 1).view(pages[0].dtype)
        pages = [both[:, 0], both[:, 1]]
        if e4m3:
            both = torch.stack(scales, 1)
            scales = [both[:, 0], both[:, 1]]
    return binding.PagedCache(*pages, *scales)


def raw(cache):
    return [t.clone().view(torch.uint8) if t.dtype != torch.uint8 else t.clone() for t in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale) if t is not None]


def places(cu, table, kv_len, page):
    """(row, page, place) of every row with a sequence."""
    got = []
    c = cu.tolist()
    for b, n in enumerate(kv_len.tolist()):
        for i in range(c[b], c[b + 1]):
            pos = n - (c[b + 1] - i)
            got.append((i, int(table[b, pos // page]), pos % page))
    return [torch.tensor(x, device="cuda") for x in zip(*got)]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("Hkv,D,page", [(4, 128, 16), (1, 64, 32), (3, 128, 64), (2, 64, 128), (5, 64, 256)])
@pytest.mark.parametrize("new,total", [([1], [1]), ([1, 0, 1, 1], [17, 0, 16, 300]), ([33, 5, 0, 250], [33, 100, 3, 251])])
def test_write_and_read_back(e4m3, Hkv, D, page, new, total):
    g = torch.Generator().manual_seed(100)
    table, n_pages = tu.scattered(g, [-(-n // page) for n in total])
    cache = make_cache(g, n_pages, Hkv, page, D, e4m3)
    n = sum(new)
    k, v = draw(g, n + 3, Hkv, D), draw(g, n + 3, Hkv, D)             # (three rows of no sequence)
    size = torch.exp2(torch.randint(-130, 110, (n + 3, Hkv, 1), generator=g).float()).cuda()
    k, v = (k.float() * size).to(torch.bfloat16), (v.float() * size.flip(0)).to(torch.bfloat16)
    k[0, 0] = 0
    cu, kv_len = tu.cumulative(new), torch.tensor(total, dtype=torch.int32, device="cuda")
    before = raw(cache)
    eng = tu.engine(2 * Hkv, Hkv, D)
    eng.paged_write(cache, k, v, cu, table, kv_len)
    ko, vo = (torch.full((n + 3, Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    eng.paged_read(cache, cu, table, kv_len, ko, vo)
    assert eng.text_status() == 0
    for got, x in ((ko, k), (vo, v)):
        assert (got[n:] == 7).all()
        if e4m3:
            want, _ = tu.quantise(x[:n])
            assert torch.equal(got[:n].double(), want)
            assert ((got[:n].double() - x[:n].double()).abs() <= torch.maximum(x[:n].double().abs() * 2.0 ** -4, x[:n].double().abs().amax(-1, keepdim=True) * 2.0 ** -17)).all()
        else:
            assert torch.equal(got[:n].view(torch.int16), x[:n].view(torch.int16))
    if n:                                                            # nothing else changed
        row, pg, pl = places(cu, table, kv_len, page)
        for was, now in zip(before, raw(cache)):
            now[pg, :, pl] = was[pg, :, pl]
            assert torch.equal(was, now)


def test_scales_and_ties_are_the_definition():
    """Rows whose largest value lies on, just above and just below 448 times a power of two, values half way between two codes."""
    D, rows = 64, []
    for top in (448.0, 450.0, 446.0, 1.75, 1.7578125, 2.0 ** -126, 2.0 ** -133, 3.0e38, 2.0 ** -120, 1.0, 0.0):
        r = torch.linspace(-1, 1, D) * top
        r[0] = top
        rows.append(r)
    r = torch.arange(D).float() / 16 + 16                            # at scale 1 the codes from 16 on are 2 apart: ties
    r[0] = 448
    rows.append(r)
    r = torch.arange(D).float() * 2.0 ** -10                         # ties between e4m3's smallest steps
    r[0] = 448
    rows.append(r)
    x = torch.stack(rows).to(torch.bfloat16).cuda()[:, None]
    n = x.shape[0]
    g = torch.Generator().manual_seed(101)
    cache = make_cache(g, 1, 1, 16, D, True)
    eng = tu.engine(1, 1, D)
    cu, kv_len, table = tu.cumulative([n]), torch.tensor([n], dtype=torch.int32, device="cuda"), torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    eng.paged_write(cache, x, x, cu, table, kv_len)
    want, byte = tu.quantise(x[:, 0])
    assert torch.equal(cache.k_scale[0, 0, :n], byte)
    assert torch.equal(tu.page_values(cache)[0][0, 0, :n], want)
    ko, vo = torch.empty_like(x), torch.empty_like(x)
    eng.paged_read(cache, cu, table, kv_len, ko, vo)
    assert torch.equal(ko[:, 0].double(), want) and torch.equal(vo, ko)


def test_values_that_are_no_numbers_are_kept_apart():
    g = torch.Generator().manual_seed(102)
    x = draw(g, 4, 1, 128)
    x[0, 0, 5], x[1, 0, 9], x[2, 0, 0] = math.inf, math.nan, -math.inf
    x[3] = math.nan
    cache = make_cache(g, 1, 1, 16, 128, True)
    eng = tu.engine(1, 1, 128)
    cu, kv_len, table = tu.cumulative([4]), torch.tensor([4], dtype=torch.int32, device="cuda"), torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    eng.paged_write(cache, x, x, cu, table, kv_len)
    got, _ = eng.paged_read(cache, cu, table, kv_len, torch.empty_like(x), torch.empty_like(x))
    want, _ = tu.quantise(x)
    assert torch.equal(torch.isnan(got), ~torch.isfinite(x))
    assert torch.equal(torch.nan_to_num(got.double(), nan=1.0), torch.nan_to_num(want, nan=1.0))


@pytest.mark.parametrize("e4m3", [False, True])
def test_rows_without_a_place_are_reported(e4m3):
    """More tokens than the table has room for, a negative position, a page that is not there: nothing is written for them, zeros are read."""
    g = torch.Generator().manual_seed(103)
    Hkv, D, page = 2, 64, 16
    cache = make_cache(g, 4, Hkv, page, D, e4m3)
    eng = tu.engine(4, Hkv, D)
    cu = tu.cumulative([3, 3, 3, 3])
    table = torch.tensor([[0], [1], [4], [-1]], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([18, 2, 3, 3], dtype=torch.int32, device="cuda")       # tokens 15 16 17 | -1 0 1 | page 4 | page -1
    k, v = draw(g, 12, Hkv, D), draw(g, 12, Hkv, D)
    before = raw(cache)
    eng.paged_write(cache, k, v, cu, table, kv_len)
    assert eng.text_status() == 1
    row, pg, pl = (torch.tensor(x, device="cuda") for x in ([0, 4, 5], [0, 1, 1], [15, 0, 1]))
    for was, now in zip(before, raw(cache)):
        now[pg, :, pl] = was[pg, :, pl]
        assert torch.equal(was, now)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    eng.paged_read(cache, cu, table, kv_len, ko, vo)
    assert eng.text_status() == 1
    lost = torch.ones(12, dtype=torch.bool, device="cuda")
    lost[row] = False
    assert (ko[lost] == 0).all() and (vo[lost] == 0).all()
    want = tu.quantise(k[row])[0] if e4m3 else k[row].double()
    assert torch.equal(ko[row].double(), want)


@pytest.mark.parametrize("e4m3", [False, True])
def test_strided_rows_and_interleaved_pages(e4m3):
    g = torch.Generator().manual_seed(104)
    Hkv, D, page, n = 4, 128, 32, 70
    table, n_pages = tu.scattered(g, [3])
    cache = make_cache(g, n_pages, Hkv, page, D, e4m3, interleaved=True)
    kv = draw(g, n, 2 * Hkv, D)
    k, v = kv[:, :Hkv], draw(g, Hkv, n, D).transpose(0, 1)
    cu, kv_len = tu.cumulative([n]), torch.tensor([n], dtype=torch.int32, device="cuda")
    eng = tu.engine(8, Hkv, D)
    eng.paged_write(cache, k, v, cu, table, kv_len)
    ko, vo = torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda"), torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda")
    eng.paged_read(cache, cu, table, kv_len, ko, vo)
    for got, x in ((ko, k), (vo, v)):
        assert torch.equal(got.double(), tu.quantise(x)[0] if e4m3 else x.double())
    q = draw(g, 1, 8, D)
    out, lse = eng.paged_decode(q, None, None, cache, table, kv_len, want_lse=True)
    want, wl, tol, ltol = tu.attend(q, ko, vo, torch.tensor([n - 1], device="cuda"), D ** -0.5)
    tu.assert_close(out, want, tol, "out")
    tu.assert_lse(lse, wl, ltol)


def filled(g, cache, table, lens, size=1.0):
    """Puts ordinary values into the tokens of the sequences, through their definition."""
    for b, n in enumerate(lens):
        for i in range(-(-n // cache.page_size)):
            pg = int(table[b, i])
            x = [draw(g, cache.n_kv_heads, cache.page_size, cache.head_dim, size=size) for _ in range(2)]
            have = min(cache.page_size, n - i * cache.page_size)
            for t, s, y in ((cache.k_pages, cache.k_scale, x[0]), (cache.v_pages, cache.v_scale, x[1])):
                if s is None:
                    t[pg, :, :have] = y[:, :have]
                else:
                    val, byte = tu.quantise(y)
                    codes = (val / torch.exp2(byte.double() - 127)[..., None]).float().to(torch.float8_e4m3fn)
                    t.view(torch.uint8)[pg, :, :have] = codes.view(torch.uint8)[:, :have]
                    s[pg, :, :have] = byte[:, :have]


def check_decode(eng, cache, table, lens, q, k_new=None, v_new=None):
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    before = raw(cache)
    out, lse = eng.paged_decode(q, k_new, v_new, cache, table, kv_len, want_lse=True)
    assert eng.text_status() == 0
    page, scale = cache.page_size, cache.head_dim ** -0.5
    after = raw(cache)
    for b, n in enumerate(lens):
        if k_new is not None and n > 0:                              # the appended token, and nothing but it
            pg, pl = int(table[b, (n - 1) // page]), (n - 1) % page
            for (val, s), x in zip(zip(tu.page_values(cache), (cache.k_scale, cache.v_scale)), (k_new, v_new)):
                want = x[b].double() if s is None else tu.quantise(x[b])[0]
                assert torch.equal(val[pg, :, pl], want)
            for was, now in zip(before, after):
                was[pg, :, pl] = now[pg, :, pl]
        if n == 0:
            assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
            continue
        kk, vv = tu.sequence_values(cache, table, b, n)
        want, wl, tol, ltol = tu.attend(q[b:b + 1], kk, vv, torch.tensor([n - 1], device="cuda"), scale)
        tu.assert_close(out[b:b + 1], want, tol, f"out of sequence {b}")
        tu.assert_lse(lse[b:b + 1], wl, ltol)
    for was, now in zip(before, after):
        assert torch.equal(was, now)
    return out, lse


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,page", [(28, 4, 128, 16), (16, 1, 64, 64), (4, 4, 64, 32), (6, 2, 128, 256), (5, 1, 128, 128), (16, 2, 64, 16), (16, 1, 128, 64), (11, 1, 128, 32)])
@pytest.mark.parametrize("lens", [[1], [2, 0, 1, 17], [64, 63, 65, 128, 129], [1000, 16, 0, 400]])
def test_decode(e4m3, append, Hq, Hkv, D, page, lens):
    """Pages hold codes of every kind behind the last token (NaN among them): no row may take anything from there."""
    g = torch.Generator().manual_seed(105)
    table, n_pages = tu.scattered(g, [-(-n // page) for n in lens])
    cache = make_cache(g, n_pages, Hkv, page, D, e4m3)
    if not e4m3:
        cache.k_pages.fill_(math.nan), cache.v_pages.fill_(math.inf)
    filled(g, cache, table, lens)
    B = len(lens)
    new = (draw(g, B, Hkv, D), draw(g, B, Hkv, D)) if append else (None, None)
    check_decode(tu.engine(Hq, Hkv, D), cache, table, lens, draw(g, B, Hq, D), *new)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("size", [0.05, 8.0])
def test_decode_long_flat_and_sharp(e4m3, size):
    g = torch.Generator().manual_seed(106)
    Hq, Hkv, D, page, lens = 28, 4, 128, 64, [20011, 3]
    table, n_pages = tu.scattered(g, [-(-n // page) for n in lens])
    cache = make_cache(g, n_pages, Hkv, page, D, e4m3)
    filled(g, cache, table, lens)
    check_decode(tu.engine(Hq, Hkv, D), cache, table, lens, draw(g, 2, Hq, D, size=size))


def test_decode_rows_of_very_different_sizes():
    """8-bit rows whose powers of two differ by tens of binades: small values with large weights beside large values with small ones."""
    g = torch.Generator().manual_seed(107)
    Hq, Hkv, D, page, n = 14, 2, 128, 32, 300
    table, n_pages = tu.scattered(g, [-(-n // page)])
    cache = make_cache(g, n_pages, Hkv, page, D, True)
    x = [draw(g, n, Hkv, D).float() for _ in range(2)]
    x[1] *= torch.exp2(torch.randint(-60, 60, (n, Hkv, 1), generator=g).float()).cuda()
    x[0] *= torch.exp2(torch.randint(-40, 1, (n, Hkv, 1), generator=g).float()).cuda()
    eng = tu.engine(Hq, Hkv, D)
    kv_len = torch.tensor([n], dtype=torch.int32, device="cuda")
    eng.paged_write(cache, x[0].to(torch.bfloat16), x[1].to(torch.bfloat16), tu.cumulative([n]), table, kv_len)
    check_decode(eng, cache, table, [n], draw(g, 1, Hq, D))
    x[1][:, :, :] = draw(g, n, Hkv, D).float() * torch.exp2(torch.where(torch.arange(n) % 2 == 0, -100.0, -30.0)).cuda()[:, None, None]
    x[0][::2] = 4.0                                                  # the small values get nearly all the weight
    x[0][1::2] = -4.0
    eng.paged_write(cache, x[0].to(torch.bfloat16), x[1].to(torch.bfloat16), tu.cumulative([n]), table, kv_len)
    check_decode(eng, cache, table, [n], torch.full((1, Hq, D), 0.5, dtype=torch.bfloat16, device="cuda"))


def test_decode_many_sequences():
    g = torch.Generator().manual_seed(108)
    Hq, Hkv, D, page = 8, 2, 64, 16
    lens = torch.randint(0, 90, (217,), generator=g).tolist()
    table, n_pages = tu.scattered(g, [-(-n // page) for n in lens])
    cache = make_cache(g, n_pages, Hkv, page, D, False)
    filled(g, cache, table, lens)
    B = len(lens)
    check_decode(tu.engine(Hq, Hkv, D), cache, table, lens, draw(g, B, Hq, D), draw(g, B, Hkv, D), draw(g, B, Hkv, D))


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_one_long_sequence_among_many(e4m3):
    """More than 32 sequences, one of them in more than 16 parts, unused slots in front and behind."""
    g = torch.Generator().manual_seed(115)
    Hq, Hkv, D, page = 14, 2, 128, 32
    lens = [0, 0] + [5] * 20 + [14001] + [70] * 20 + [0]
    table, n_pages = tu.scattered(g, [-(-n // page) for n in lens])
    cache = make_cache(g, n_pages, Hkv, page, D, e4m3)
    filled(g, cache, table, lens)
    B = len(lens)
    check_decode(tu.engine(Hq, Hkv, D), cache, table, lens, draw(g, B, Hq, D), draw(g, B, Hkv, D), draw(g, B, Hkv, D))


def test_decode_values_that_are_no_numbers():
    """A key that is no number makes its sequence's rows none; an infinite value reaches its own coordinate; other sequences keep theirs."""
    g = torch.Generator().manual_seed(116)
    Hq, Hkv, D, page, lens = 8, 2, 128, 16, [200, 90, 40]
    table, n_pages = tu.scattered(g, [-(-n // page) for n in lens])
    cache = make_cache(g, n_pages, Hkv, page, D, False)
    filled(g, cache, table, lens)
    eng = tu.engine(Hq, Hkv, D)
    q, kv_len = draw(g, 3, Hq, D), torch.tensor(lens, dtype=torch.int32, device="cuda")
    clean, _ = eng.paged_decode(q, None, None, cache, table, kv_len)
    cache.k_pages[int(table[0, 3]), 0, 2, 7] = math.nan
    cache.v_pages[int(table[1, 2]), 1, 5, 9] = math.inf
    out, _ = eng.paged_decode(q, None, None, cache, table, kv_len)
    assert torch.isnan(out[0, :4]).all() and torch.equal(out[0, 4:], clean[0, 4:])
    assert (out[1, 4:, 9] == math.inf).all() and torch.equal(out[1, :4], clean[1, :4])
    others = [i for i in range(D) if i != 9]
    assert torch.equal(out[1, 4:][:, others], clean[1, 4:][:, others]) and torch.equal(out[2], clean[2])


@pytest.mark.parametrize("e4m3", [False, True])
def test_what_the_workspace_held_does_not_matter(e4m3):
    g = torch.Generator().manual_seed(117)
    Hq, Hkv, D, page, lens = 14, 2, 64, 64, [3000, 0, 100, 2000]
    table, n_pages = tu.scattered(g, [-(-n // page) for n in lens])
    cache = make_cache(g, n_pages, Hkv, page, D, e4m3)
    filled(g, cache, table, lens)
    eng, q = tu.engine(Hq, Hkv, D), draw(g, 4, Hq, D)
    out, lse = check_decode(eng, cache, table, lens, q)
    eng._text_ws.fill_(255)
    again, lse2 = check_decode(eng, cache, table, lens, q)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_only_unused_slots():
    g = torch.Generator().manual_seed(118)
    cache = make_cache(g, 3, 2, 16, 64, False)
    check_decode(tu.engine(4, 2, 64), cache, torch.zeros(3, 2, dtype=torch.int32, device="cuda"), [0, 0, 0], draw(g, 3, 4, 64), draw(g, 3, 2, 64), draw(g, 3, 2, 64))


def test_first_call_inside_a_capture_is_refused():
    eng = tu.engine(4, 2, 64)
    cache = eng.paged_cache(4, 16)
    q, table, kv_len = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    g, x = torch.cuda.CUDAGraph(), torch.zeros(1, device="cuda")
    with torch.cuda.graph(g):
        x.add_(1)
        with pytest.raises(binding.AdasparkError):
            eng.paged_decode(q, None, None, cache, table, kv_len, out=out)
    eng.paged_decode(q, None, None, cache, table, kv_len, out=out)
    assert eng.text_status() == 0


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_shared_pages_and_strided_rows(e4m3):
    """Two sequences with the same first pages; queries and new rows as slices of a fused projection."""
    g = torch.Generator().manual_seed(109)
    Hq, Hkv, D, page = 16, 4, 64, 16
    table = torch.tensor([[3, 1, 0], [3, 1, 2]], dtype=torch.int32, device="cuda")
    cache = make_cache(g, 5, Hkv, page, D, e4m3)
    lens = [40, 47]
    filled(g, cache, table, lens)
    x = draw(g, 2, Hq + 2 * Hkv, D)
    check_decode(tu.engine(Hq, Hkv, D), cache, table, lens, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])


def test_decode_bad_pages_and_lengths_are_reported():
    g = torch.Generator().manual_seed(110)
    Hq, Hkv, D, page = 8, 2, 128, 16
    cache = make_cache(g, 4, Hkv, page, D, False)
    eng = tu.engine(Hq, Hkv, D)
    q, kn, vn = draw(g, 5, Hq, D), draw(g, 5, Hkv, D), draw(g, 5, Hkv, D)
    table = torch.tensor([[0, 1], [2, 9], [3, 0], [3, 0], [-4, 1]], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([20, 20, 33, -1, 3], dtype=torch.int32, device="cuda")   # good | page 9 | beyond the table | negative | page -4
    before = raw(cache)
    out, lse = eng.paged_decode(q, kn, vn, cache, table, kv_len, want_lse=True)
    assert eng.text_status() == 1
    assert (out[1:] == 0).all() and (lse[1:] == -math.inf).all()
    for was, now in zip(before, raw(cache)):
        now[1, :, 3] = was[1, :, 3]
        assert torch.equal(was, now)
    kk, vv = tu.sequence_values(cache, table, 0, 20)
    want, wl, tol, ltol = tu.attend(q[:1], kk, vv, torch.tensor([19], device="cuda"), D ** -0.5)
    tu.assert_close(out[:1], want, tol, "out")


def test_captured_decode_steps():
    """A captured step replayed while lengths, tables and inputs change, two graphs on one workspace one after the other."""
    g = torch.Generator().manual_seed(111)
    Hq, Hkv, D, page = 28, 4, 128, 16
    lens = [30, 100, 7]
    table, n_pages = tu.scattered(g, [10, 10, 10])
    cache = make_cache(g, n_pages, Hkv, page, D, True)
    filled(g, cache, table, lens)
    eng = tu.engine(Hq, Hkv, D)
    q, kn, vn = draw(g, 3, Hq, D), draw(g, 3, Hkv, D), draw(g, 3, Hkv, D)
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = eng.paged_decode(q, None, None, cache, table, kv_len, want_lse=True)
    out2 = torch.empty_like(out)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        eng.paged_decode(q, kn, vn, cache, table, kv_len, out=out, lse=lse)
    with torch.cuda.graph(graphs[1]):
        eng.paged_decode(q, None, None, cache, table, kv_len, out=out2, lse=lse)
    for step in range(4):
        for t in (q, kn, vn):
            t.copy_(draw(g, *t.shape))
        kv_len += 1
        out.zero_(), out2.zero_()
        graphs[0].replay()
        graphs[1].replay()
        assert torch.equal(out, out2)
        for b in range(3):
            n = lens[b] + step + 1
            kk, vv = tu.sequence_values(cache, table, b, n)
            assert torch.equal(kk[n - 1], tu.quantise(kn[b])[0])
            want, wl, tol, ltol = tu.attend(q[b:b + 1], kk, vv, torch.tensor([n - 1], device="cuda"), D ** -0.5)
            tu.assert_close(out[b:b + 1], want, tol, "out")
            tu.assert_lse(lse[b:b + 1], wl, ltol)
    assert eng.text_status() == 0


def test_pool_of_more_than_2_31_elements():
    """Pages whose offsets need more than 32 bits, at the end of a pool of 2.2 G codes."""
    Hkv, D, page = 4, 128, 64
    n_pages = (1 << 31) // (Hkv * D * page) + 2000
    k = torch.zeros(n_pages, Hkv, page, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros(n_pages, Hkv, page, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    s = [torch.zeros(n_pages, Hkv, page, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = binding.PagedCache(k, v, *s)
    g = torch.Generator().manual_seed(112)
    n = 200
    x = draw(g, n, 2 * Hkv, D)
    table = torch.tensor([[n_pages - 1, 5, n_pages - 3, n_pages - 2]], dtype=torch.int32, device="cuda")
    kv_len, cu = torch.tensor([n], dtype=torch.int32, device="cuda"), tu.cumulative([n])
    eng = tu.engine(8, Hkv, D)
    eng.paged_write(cache, x[:, :Hkv], x[:, Hkv:], cu, table, kv_len)
    ko, vo = torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda"), torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda")
    eng.paged_read(cache, cu, table, kv_len, ko, vo)
    want = [tu.quantise(y)[0] for y in (x[:, :Hkv], x[:, Hkv:])]
    assert torch.equal(ko.double(), want[0]) and torch.equal(vo.double(), want[1])
    q, kn, vn = draw(g, 1, 8, D), draw(g, 1, Hkv, D), draw(g, 1, Hkv, D)
    kv_len += 1
    out, lse = eng.paged_decode(q, kn, vn, cache, table, kv_len, want_lse=True)
    kk, vv = (torch.cat([a, tu.quantise(b)[0]]) for a, b in zip(want, (kn, vn)))
    ref, wl, tol, ltol = tu.attend(q, kk, vv, torch.tensor([n], device="cuda"), D ** -0.5)
    tu.assert_close(out, ref, tol, "out")
    tu.assert_lse(lse, wl, ltol)


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_conversation(e4m3):
    """The operators as they are used together: prompts of two requests are written to the cache and attended, tokens follow one by
    one, one request goes on with a second prompt whose earlier tokens are read back, and every output is what the whole sequence gives."""
    g = torch.Generator().manual_seed(113)
    Hq, Hkv, D, page = 28, 4, 128, 16
    eng = tu.engine(Hq, Hkv, D)
    cache = eng.paged_cache(40, page, e4m3=e4m3)
    table = torch.randperm(40, generator=g).to(torch.int32).view(2, 20).cuda()
    lens = [150, 61]
    held = [[], []]                                                  # (k, v) rows as the cache holds them
    kept = lambda x: tu.quantise(x)[0] if e4m3 else x.double()       # noqa: E731
    x = draw(g, sum(lens), Hq + 2 * Hkv, D)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    cu, kv_len = tu.cumulative(lens), torch.tensor(lens, dtype=torch.int32, device="cuda")
    eng.paged_write(cache, k, v, cu, table, kv_len)
    out, _ = eng.prompt(q, k, v, cu)                                 # a fresh prompt attends its own keys, not yet rounded
    mine, want, _, tol, _ = tu.prompt_reference(q, k, v, cu, cu, D ** -0.5)
    tu.assert_close(out, want, tol, "prompt")
    at = 0
    for b, n in enumerate(lens):
        held[b] = [kept(k[at:at + n]), kept(v[at:at + n])]
        at += n
    for step in range(3):
        kv_len += 1
        q, kn, vn = draw(g, 2, Hq, D), draw(g, 2, Hkv, D), draw(g, 2, Hkv, D)
        out, lse = eng.paged_decode(q, kn, vn, cache, table, kv_len, want_lse=True)
        for b in range(2):
            held[b] = [torch.cat([a, kept(y[b:b + 1])]) for a, y in zip(held[b], (kn, vn))]
            n = held[b][0].shape[0]
            want, wl, tol, ltol = tu.attend(q[b:b + 1], *held[b], torch.tensor([n - 1], device="cuda"), D ** -0.5)
            tu.assert_close(out[b:b + 1], want, tol, "decode")
            tu.assert_lse(lse[b:b + 1], wl, ltol)
    new = 45                                                         # the second turn of request 0
    q, kn, vn = draw(g, new, Hq, D), draw(g, new, Hkv, D), draw(g, new, Hkv, D)
    kv_len[0] += new
    total = int(kv_len[0])
    eng.paged_write(cache, kn, vn, tu.cumulative([new]), table[:1], kv_len[:1])
    ko, vo = torch.empty(total, Hkv, D, dtype=torch.bfloat16, device="cuda"), torch.empty(total, Hkv, D, dtype=torch.bfloat16, device="cuda")
    eng.paged_read(cache, tu.cumulative([total]), table[:1], kv_len[:1], ko, vo)
    out, _ = eng.prompt(q, ko, vo, tu.cumulative([new]), tu.cumulative([total]))
    full = [torch.cat([a, kept(y)]) for a, y in zip(held[0], (kn, vn))]
    want, _, tol, _ = tu.attend(q, *full, torch.arange(new, device="cuda") + total - new, D ** -0.5)
    tu.assert_close(out, want, tol, "second turn")
    assert eng.text_status() == 0


def test_refusals():
    eng = tu.engine(4, 2, 64)
    cache, other = eng.paged_cache(4, 16), tu.engine(4, 4, 64).paged_cache(4, 16)
    g = torch.Generator().manual_seed(114)
    q, k, v = draw(g, 2, 4, 64), draw(g, 2, 2, 64), draw(g, 2, 2, 64)
    table, kv_len, cu = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda"), tu.cumulative([1, 1])
    for bad in [(q, k, None, cache, table, kv_len), (q, k, v, other, table, kv_len), (q[:1], k, v, cache, table, kv_len), (q, k, v, cache, table[:1], kv_len),
                (q, k, v, cache, table.long(), kv_len), (q.float(), k, v, cache, table, kv_len), (q, k, v, cache, table, kv_len.cpu())]:
        with pytest.raises(binding.AdasparkError):
            eng.paged_decode(*bad)
    for bad in [(cache, k, v[:1], cu, table, kv_len), (cache, k, v, cu[:2], table, kv_len), (other, k, v, cu, table, kv_len), (cache, q, v, cu, table, kv_len)]:
        with pytest.raises(binding.AdasparkError):
            eng.paged_write(*bad)
    with pytest.raises(binding.AdasparkError):
        eng.paged_read(cache, cu, table, kv_len, k, v.float())
