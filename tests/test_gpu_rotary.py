"""Norms and rotated positions of queries and keys, as rows and on the way into a paged cache, against 64 bits."""
import pytest
import torch

from paper_2604_08077_b200 import binding
from text_util import BF16_HALF, assert_close, cumulative, engine, page_values, scattered
from window_util import rotated

pytestmark = pytest.mark.gpu
EPS = 1e-6


def rand(g, *shape, scale=1.0):
    return (scale * torch.randn(*shape, generator=g)).to(torch.bfloat16).cuda()


def turn(D, sections, adjacent, theta=1e4):
    n = sum(sections)
    return (binding.Rotary(D, sections=sections, theta=theta, adjacent=adjacent), [theta ** (-i / n) for i in range(n)],
            [a for a, m in enumerate(sections) for _ in range(m)])


def check(got, x, weight, positions, freq, axis, adjacent, what, eps=EPS):
    want, tol = rotated(x, weight, positions, freq, axis, adjacent, eps)
    assert_close(got, want, tol + BF16_HALF * want.abs() + 1e-30, what)


@pytest.mark.parametrize("Hq,Hkv,D,n,sections,adjacent,norm", [
    (28, 4, 128, 1, [16, 24, 24], False, True), (28, 4, 128, 37, [64], False, False), (28, 4, 128, 1025, [16, 24, 24], True, True),
    (28, 4, 128, 1024, [8, 8], False, True), (4, 4, 64, 3, [32], True, False), (16, 4, 64, 2049, [8], False, True), (16, 4, 64, 701, [16], True, False),
    (8, 2, 128, 130, [16, 16, 16, 16], False, True), (1, 1, 64, 9, [8, 12, 12], False, True), (16, 1, 128, 1030, [40], True, True)])
def test_rotate(Hq, Hkv, D, n, sections, adjacent, norm):
    g = torch.Generator().manual_seed(n)
    eng = engine(Hq, Hkv, D)
    r, freq, axis = turn(D, sections, adjacent)
    q, k = rand(g, n, Hq, D, scale=3.0), rand(g, n, Hkv, D)
    wq, wk = (rand(g, D), rand(g, D)) if norm else (None, None)
    pos = torch.randint(-5, 140000, (len(sections), n), generator=g, dtype=torch.int32).cuda()
    qo, ko = eng.rotate(q, k, pos, r, q_norm=wq, k_norm=wk, eps=EPS)
    check(qo, q, wq, pos, freq, axis, adjacent, "q")
    check(ko, k, wk, pos, freq, axis, adjacent, "k")


def test_rows_where_they_are():
    """Slices of a fused projection, turned in place; what lies beside them stays."""
    g = torch.Generator().manual_seed(5)
    Hq, Hkv, D, n = 8, 2, 128, 77
    eng = engine(Hq, Hkv, D)
    r, freq, axis = turn(D, [64], False)
    qkv = rand(g, n, Hq + 2 * Hkv, D)
    before = qkv.clone()
    pos = torch.arange(n, dtype=torch.int32).cuda()
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
    got = eng.rotate(q, k, pos, r, q_out=q, k_out=k)
    assert got[0] is q and got[1] is k
    check(q, before[:, :Hq], None, pos, freq, axis, False, "q")
    check(k, before[:, Hq:Hq + Hkv], None, pos, freq, axis, False, "k")
    assert torch.equal(qkv[:, Hq + Hkv:], before[:, Hq + Hkv:])
    heads_first = rand(g, Hq, n, D)
    qo, none = eng.rotate(heads_first.transpose(0, 1), None, pos, r)
    assert none is None
    check(qo, heads_first.transpose(0, 1), None, pos, freq, axis, False, "q of head-major rows")


def test_far_positions():
    g = torch.Generator().manual_seed(6)
    eng = engine(4, 4, 64)
    r, freq, axis = turn(64, [32], False, theta=1e6)
    pos = torch.tensor([2 ** 31 - 1, -2 ** 31, -1, 0, 1, 2 ** 30 + 12345, 999999999], dtype=torch.int32).cuda()
    q = rand(g, pos.numel(), 4, 64)
    qo, _ = eng.rotate(q, None, pos, r)
    # 64-bit products of a position and a frequency are off by 2^-53 of up to 2^31: 2^-22 of a radian, and so is the fraction of a turn's frequency
    want, tol = rotated(q, None, pos, freq, axis, False, EPS)
    assert_close(qo, want, tol + BF16_HALF * want.abs() + q.double().abs().amax() * 2.0 ** -20, "far positions")
    assert torch.equal(qo[3], q[3])


def test_small_angles_beside_zeros():
    """A pair (0, b) gives -b sin t: relative to itself as exact as any."""
    eng = engine(4, 4, 64)
    r, freq, axis = turn(64, [32], False, theta=1e9)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    q[..., 32:] = 1.5
    pos = torch.tensor([1, -7, 100], dtype=torch.int32).cuda()
    qo, _ = eng.rotate(q, None, pos, r)
    want, _ = rotated(q, None, pos, freq, axis, False, EPS)
    assert_close(qo, want, want.abs() * (BF16_HALF + 2.0 ** -20) + 1e-30, "small angles")


def test_own_frequencies_and_interleaved_axes():
    g = torch.Generator().manual_seed(8)
    eng = engine(4, 2, 128)
    freq = [0.9 ** i if i % 3 else -7.5 for i in range(48)]
    axis = [i % 3 for i in range(48)]
    r = binding.Rotary(128, frequencies=freq, axis=axis)
    q, k, pos = rand(g, 19, 4, 128), rand(g, 19, 2, 128), torch.randint(0, 500, (3, 19), generator=g, dtype=torch.int32).cuda()
    qo, ko = eng.rotate(q, k, pos, r)
    check(qo, q, None, pos, freq, axis, False, "q")
    check(ko, k, None, pos, freq, axis, False, "k")


@pytest.mark.parametrize("D,adjacent", [(128, False), (64, True)])
def test_as_many_tokens_as_a_long_video_has(D, adjacent):
    g = torch.Generator().manual_seed(15)
    Hq, Hkv, n, page = 2, 1, 33001, 64
    eng = engine(Hq, Hkv, D)
    r, freq, axis = turn(D, [8, 8, 8], adjacent)
    q, k, v, w = rand(g, n, Hq, D), rand(g, n, Hkv, D), rand(g, n, Hkv, D), rand(g, D)
    pos = torch.randint(0, 1000, (3, n), generator=g, dtype=torch.int32).cuda()
    qo, ko = eng.rotate(q, k, pos, r, q_norm=w)
    check(qo, q, w, pos, freq, axis, adjacent, "q")
    check(ko, k, None, pos, freq, axis, adjacent, "k")
    table, cache = pool(g, [n], page, Hkv, D, False)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    qa = eng.paged_append(cache, q, k, v, cumulative([n]), table, lens, r, positions=pos, q_norm=w)
    got = [x[table[0].long()].transpose(1, 2).reshape(-1, Hkv, D)[:n] for x in (cache.k_pages, cache.v_pages)]
    assert torch.equal(qa, qo) and torch.equal(got[0], ko) and torch.equal(got[1], v)


def test_norm_alone_and_sizes_whose_squares_leave_32_bits():
    g = torch.Generator().manual_seed(9)
    eng = engine(4, 4, 128)
    w = rand(g, 128)
    size = torch.exp2(torch.tensor([-100.0, -20.0, 0.0, 62.0, 64.0, 100.0, 120.0]))[:, None, None]
    q = (torch.randn(7, 4, 128, generator=g) * size).to(torch.bfloat16).cuda()
    qo, _ = eng.rotate(q, None, q_norm=w, eps=1e-5)
    check(qo, q, w, None, [], [], False, "norm", eps=1e-5)
    same, _ = eng.rotate(q, None)
    assert torch.equal(same, q)
    zeros, _ = eng.rotate(torch.zeros_like(q), None, q_norm=w)
    assert torch.equal(zeros, torch.zeros_like(q))


def test_norm_beside_values_that_are_no_numbers():
    g = torch.Generator().manual_seed(91)
    eng = engine(4, 4, 64)
    w, q = rand(g, 64), rand(g, 3, 4, 64)
    q[0, 1, 5], q[1, 0, 63], q[1, 0, 2], q[2, 3, 7] = float("inf"), float("-inf"), float("inf"), float("nan")
    qo, _ = eng.rotate(q, None, q_norm=w)
    x = q.double()
    want = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.double()
    assert torch.equal(qo.isnan(), want.isnan()) and want.isnan().sum() == 67
    assert (qo[0, 1][torch.arange(64) != 5] == 0).all()
    rest = torch.ones(3, 4, dtype=torch.bool)
    rest[0, 1] = rest[1, 0] = rest[2, 3] = False
    check(qo[rest][None], q[rest][None], w, None, [], [], False, "rows beside them", eps=1e-6)


def pages_of(cache):
    """Pages and powers of two as bytes."""
    return [x.view(torch.uint8) for x in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale) if x is not None]


def test_no_rows():
    eng = engine(4, 2, 64)
    r, _, _ = turn(64, [32], False)
    q, k = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.empty(0, dtype=torch.int32, device="cuda")
    qo, ko = eng.rotate(q, k, pos, r)
    assert qo.shape == q.shape and ko.shape == k.shape


# ---------------------------------------------------------------------------------------------------------------- into pages

def pool(g, lens, page, Hkv, D, e4m3):
    table, n_pages = scattered(g, [-(-n // page) for n in lens])
    shape = (n_pages, Hkv, page, D)
    if not e4m3:
        return table, binding.PagedCache(rand(g, *shape), rand(g, *shape))
    codes = [torch.randint(0, 127, shape, generator=g, dtype=torch.uint8).cuda().view(torch.float8_e4m3fn) for _ in range(2)]
    return table, binding.PagedCache(*codes, *(torch.randint(100, 130, shape[:3], generator=g, dtype=torch.uint8).cuda() for _ in range(2)))


def places(table, kv_len, cu, page):
    got = []
    for b, n in enumerate(kv_len):
        for i in range(cu[b + 1] - cu[b]):
            pos = n - (cu[b + 1] - cu[b]) + i
            got.append((cu[b] + i, int(table[b, pos // page]), pos % page, pos))
    return got


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,page,new,ctx,sections,adjacent,norm,own_positions", [
    (28, 4, 128, 64, [1] * 5, [131, 0, 63, 64, 1000], [16, 24, 24], False, True, True),
    (16, 4, 64, 16, [700, 0, 1, 33, 16], [0, 5, 15, 100, 48], [32], False, True, False),
    (28, 4, 128, 16, [1100, 17], [3, 0], [64], True, False, False),
    (8, 2, 128, 256, [300, 1], [0, 255], [16], False, True, True),
    (4, 4, 64, 32, [9, 2], [0, 31], [], False, False, False)])
def test_append(Hq, Hkv, D, page, new, ctx, sections, adjacent, norm, own_positions, e4m3):
    g = torch.Generator().manual_seed(sum(new))
    eng = engine(Hq, Hkv, D)
    kv_len = [a + b if a else 0 for a, b in zip(new, ctx)]
    table, cache = pool(g, kv_len, page, Hkv, D, e4m3)
    cu_t = cumulative(new, first=2)
    cu, n = cu_t.tolist(), sum(new) + 5                          # two rows in front, three behind
    q, k, v = rand(g, n, Hq, D), rand(g, n, Hkv, D, scale=2.0), rand(g, n, Hkv, D)
    k[3] = 0
    wq, wk = (rand(g, D), rand(g, D)) if norm else (None, None)
    r, freq, axis = turn(D, sections, adjacent) if sections else (None, [], [])
    pos = torch.randint(0, 200000, (max(len(sections), 1), n), generator=g, dtype=torch.int32).cuda() if own_positions else None
    before = page_values(cache)
    q_out = rand(g, n, Hq, D)
    kept = q_out.clone()
    lens = torch.tensor(kv_len, dtype=torch.int32, device="cuda")
    got = eng.paged_append(cache, q, k, v, cu_t, table, lens, r, positions=pos, q_norm=wq, k_norm=wk, eps=EPS, q_out=q_out)
    assert got is q_out and eng.text_status() == 0
    where = places(table, kv_len, cu, page)
    rows = torch.tensor([x[0] for x in where], device="cuda")
    used = pos[:, rows] if pos is not None else torch.tensor([x[3] for x in where], device="cuda").expand(max(len(sections), 1), len(where))
    check(q_out[rows], q[rows], wq, used, freq, axis, adjacent, "q")
    assert torch.equal(q_out[:2], kept[:2]) and torch.equal(q_out[cu[-1]:], kept[cu[-1]:])
    want_k, tol_k = rotated(k[rows], wk, used, freq, axis, adjacent, EPS)
    at = (torch.tensor([x[1] for x in where], device="cuda"), slice(None), torch.tensor([x[2] for x in where], device="cuda"))
    after = page_values(cache)
    for got, old, want, tol, scales, what in ((after[0], before[0], want_k, tol_k, cache.k_scale, "k"), (after[1], before[1], v[rows].double(), 0 * tol_k, cache.v_scale, "v")):
        if e4m3:
            # half a step of four significant bits, 2^-4 of a value, or half of the smallest step, 2^-10 of the power of two: the smallest one
            # that holds the row, or the next where the largest value is as near to its limit as `tol`
            top = want.abs().amax(-1)
            s = scales[at].double() - 127
            assert (top <= 448 * torch.exp2(s) + tol.amax(-1)).all()
            assert ((top >= 448 * torch.exp2(s - 1) - tol.amax(-1)) | (s == -127)).all()
            tol = tol + want.abs() * 2.0 ** -4 + (2.0 ** -10 * torch.exp2(s))[..., None]
        elif what == "k":
            tol = tol + BF16_HALF * want.abs()
        assert_close(got[at], want, tol + 1e-30, what)
        old = old.clone()
        old[at] = got[at]
        assert torch.equal(old, got), f"{what}: other places"


@pytest.mark.parametrize("D,n", [(128, 50), (64, 1500)])
def test_bf16_pages_are_rotate_and_write(D, n):
    g = torch.Generator().manual_seed(11)
    Hq, Hkv, page = 8, 2, 32
    eng = engine(Hq, Hkv, D)
    table, a = pool(g, [n], page, Hkv, D, False)
    b = binding.PagedCache(a.k_pages.clone(), a.v_pages.clone())
    q, k, v, w = rand(g, n, Hq, D), rand(g, n, Hkv, D), rand(g, n, Hkv, D), rand(g, D)
    cu, lens = cumulative([n]), torch.tensor([n], dtype=torch.int32, device="cuda")
    r, _, _ = turn(D, [D // 2], False)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    qa = eng.paged_append(a, q, k, v, cu, table, lens, r, q_norm=w, k_norm=w)
    qb, kb = eng.rotate(q, k, pos, r, q_norm=w, k_norm=w)
    eng.paged_write(b, kb, v, cu, table, lens)
    assert torch.equal(qa, qb) and torch.equal(a.k_pages, b.k_pages) and torch.equal(a.v_pages, b.v_pages)
    c = binding.PagedCache(torch.zeros_like(a.k_pages), torch.zeros_like(a.v_pages))
    assert eng.paged_append(c, None, k, v, cu, table, lens, r, k_norm=w) is None
    eng.paged_append(a, q, k, v, cu, table, lens, r, q_norm=w, k_norm=w)          # the same again
    used = table[0, :-(-n // page)].long()
    got = [x[used].transpose(1, 2).reshape(-1, Hkv, D)[:n] for x in (a.k_pages, c.k_pages)]
    assert torch.equal(*got)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("D,n,pieces", [(128, 32800, [200, 299, 301, 2000, 30000]), (64, 6200, [100, 599, 601, 4900]), (128, 2500, [1, 2499])])
def test_in_one_call_or_in_several(D, n, pieces, e4m3):
    """The same rows whatever number of tokens a call has."""
    g = torch.Generator().manual_seed(n)
    Hq, Hkv, page = 3, 1, 32
    assert sum(pieces) == n
    eng = engine(Hq, Hkv, D)
    r, _, _ = turn(D, [8, 16], True)
    q, k, v, w = rand(g, n, Hq, D), rand(g, n, Hkv, D), rand(g, n, Hkv, D), rand(g, D)
    pos = torch.randint(0, 100000, (2, n), generator=g, dtype=torch.int32).cuda()
    table, one = pool(g, [n], page, Hkv, D, e4m3)
    other = binding.PagedCache(*(x.clone() for x in (one.k_pages, one.v_pages, one.k_scale, one.v_scale) if x is not None))
    got = eng.paged_append(one, q, k, v, cumulative([n]), table, torch.tensor([n], dtype=torch.int32, device="cuda"), r, positions=pos, q_norm=w, k_norm=w)
    turned, _ = eng.rotate(q, None, pos, r, q_norm=w)
    assert torch.equal(got, turned)
    at = 0
    for m in pieces:
        rows = slice(at, at + m)
        at += m
        part = eng.paged_append(other, q[rows], k[rows], v[rows], cumulative([m]), table, torch.tensor([at], dtype=torch.int32, device="cuda"), r,
                                positions=pos[:, rows].contiguous(), q_norm=w, k_norm=w)
        assert torch.equal(part, got[rows])
    assert eng.text_status() == 0
    for a, b in zip(pages_of(one), pages_of(other)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("Hq,Hkv,D,n", [(28, 4, 128, 77), (16, 4, 64, 4100)])
def test_append_of_a_fused_projection_in_place(Hq, Hkv, D, n):
    """q, k and v are slices of one tensor, and q comes back where it was."""
    g = torch.Generator().manual_seed(121)
    eng = engine(Hq, Hkv, D)
    r, _, _ = turn(D, [D // 2], False)
    qkv, w = rand(g, n, Hq + 2 * Hkv, D), rand(g, D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    table, a = pool(g, [n], 16, Hkv, D, False)
    b = binding.PagedCache(a.k_pages.clone(), a.v_pages.clone())
    cu, lens, before = cumulative([n]), torch.tensor([n], dtype=torch.int32, device="cuda"), qkv.clone()
    want = eng.paged_append(a, q, k, v, cu, table, lens, r, q_norm=w, k_norm=w)
    assert torch.equal(qkv, before)
    assert eng.paged_append(b, q, k, v, cu, table, lens, r, q_norm=w, k_norm=w, q_out=q) is q
    assert torch.equal(q, want) and torch.equal(qkv[:, Hq:], before[:, Hq:])
    assert torch.equal(a.k_pages, b.k_pages) and torch.equal(a.v_pages, b.v_pages)
    # heads in front of tokens
    c = binding.PagedCache(torch.zeros_like(a.k_pages), torch.zeros_like(a.v_pages))
    qt, kt, vt = (before[:, x].transpose(0, 1).contiguous().transpose(0, 1) for x in (slice(0, Hq), slice(Hq, Hq + Hkv), slice(Hq + Hkv, None)))
    assert torch.equal(eng.paged_append(c, qt, kt, vt, cu, table, lens, r, q_norm=w, k_norm=w), want)
    used = table[0].long()
    assert torch.equal(c.k_pages[used].transpose(1, 2).reshape(-1, Hkv, D)[:n], a.k_pages[used].transpose(1, 2).reshape(-1, Hkv, D)[:n])


@pytest.mark.parametrize("e4m3", [False, True])
def test_append_of_rows_without_a_place(e4m3):
    """Bad pages, lengths and bounds: reported, not followed; everything else is done."""
    g = torch.Generator().manual_seed(12)
    Hq, Hkv, D, page = 4, 2, 64, 16
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, [32] * 6, page, Hkv, D, e4m3)
    table[1, 1] = cache.n_pages
    table[2, 0] = -1
    kv_len = torch.tensor([20, 20, 20, 33, 3, 16], dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, 6, 12, 18, 24, 30, 99], dtype=torch.int32, device="cuda")       # the last one leaves the tensors
    n = 36
    q, k, v = rand(g, n, Hq, D), rand(g, n, Hkv, D), rand(g, n, Hkv, D)
    before = [x.clone() for x in (cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8))]
    q_out = eng.paged_append(cache, q, k, v, cu, table, kv_len)
    assert eng.text_status() == 1 and eng.text_status() == 0
    # sequence 0 whole; 1: its tokens 14, 15 have a place, 16 .. 19 none; 2: 16 .. have one, 14, 15 none; 3: 27 .. 31, token 32 not; 4: the last three rows
    there = torch.tensor([True] * 6 + [True] * 2 + [False] * 4 + [False] * 2 + [True] * 4 + [True] * 5 + [False] + [False] * 3 + [True] * 3 + [False] * 6, device="cuda")
    assert torch.equal(q_out, torch.where(there[:, None, None], q, 0))
    written = sum((x != y).any(-1).any(1).sum().item() for x, y in zip((cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8)), before))
    assert written == 2 * int(there.sum())


def test_values_that_are_no_numbers_in_8_bits():
    g = torch.Generator().manual_seed(13)
    eng = engine(4, 2, 64)
    cache = eng.paged_cache(4, 16, e4m3=True)
    table = torch.tensor([[2]], dtype=torch.int32, device="cuda")
    k, v = rand(g, 3, 2, 64), rand(g, 3, 2, 64)
    k[0, 0, 5], v[1, 1, 7], k[2, 1, 0] = float("inf"), float("nan"), float("-inf")
    cu, lens = cumulative([3]), torch.tensor([3], dtype=torch.int32, device="cuda")
    eng.paged_append(cache, None, k, v, cu, table, lens)
    ref = eng.paged_cache(4, 16, e4m3=True)
    eng.paged_write(ref, k, v, cu, table, lens)
    for a, b in ((cache.k_pages, ref.k_pages), (cache.v_pages, ref.v_pages)):
        a, b = a.float(), b.float()
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())
    assert torch.equal(cache.k_scale, ref.k_scale) and torch.equal(cache.v_scale, ref.v_scale)


@pytest.mark.parametrize("batch", [31, 32, 100])
def test_append_of_many_sequences(batch):
    """Places found by the lanes of a warp, and by a search; sequences without rows among them."""
    g = torch.Generator().manual_seed(batch)
    Hq, Hkv, D, page = 4, 2, 64, 16
    eng = engine(Hq, Hkv, D)
    new = [int(x) for x in torch.randint(0, 40, (batch,), generator=g)]
    kv_len = [a + int(x) for a, x in zip(new, torch.randint(0, 50, (batch,), generator=g))]
    table, cache = pool(g, kv_len, page, Hkv, D, False)
    n = sum(new)
    q, k, v = rand(g, n, Hq, D), rand(g, n, Hkv, D), rand(g, n, Hkv, D)
    cu = cumulative(new)
    eng.paged_append(cache, q, k, v, cu, table, torch.tensor(kv_len, dtype=torch.int32, device="cuda"))
    assert eng.text_status() == 0
    where = places(table, kv_len, cu.tolist(), page)
    rows, pages, slots = (torch.tensor([x[i] for x in where], device="cuda") for i in range(3))
    assert torch.equal(cache.k_pages[pages, :, slots], k[rows]) and torch.equal(cache.v_pages[pages, :, slots], v[rows])
