"""GPU tests of causal attention over packed prompts against a plain form in 64 bits."""
import math

import pytest
import torch

import text_util as tu
from paper_2604_08077_b200 import binding

pytestmark = pytest.mark.gpu


def draw(seed, n, heads, D, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, heads, D, generator=g) * size).to(torch.bfloat16).cuda()


def check(Hq, Hkv, D, q, k, v, cu_q, cu_k, softmax_scale=0.0):
    eng = tu.engine(Hq, Hkv, D, softmax_scale=softmax_scale)
    out = torch.full((q.shape[0], Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((q.shape[0], Hq), 7.0, dtype=torch.float32, device="cuda")
    got = eng.prompt(q, k, v, cu_q, cu_k, out=out, lse=lse)
    assert got[0] is out and got[1] is lse and eng.text_status() == 0
    mine, want, want_lse, tol, ltol = tu.prompt_reference(q, k, v, cu_q, cu_q if cu_k is None else cu_k, softmax_scale or D ** -0.5)
    tu.assert_close(out[mine], want[mine], tol[mine], "out")
    tu.assert_lse(lse[mine], want_lse[mine], ltol[mine])
    assert (out[~mine] == 7).all() and (lse[~mine] == 7).all(), "rows of no sequence were written"
    return out, lse


HEADS = [(4, 4, 64), (16, 4, 64), (28, 4, 128), (16, 1, 128), (6, 2, 64), (5, 1, 128), (26, 2, 128), (2, 2, 128)]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("lens", [[1], [2, 1], [0, 1, 0, 5, 0], [127, 1, 130], [36, 37, 35, 18, 17, 19], [300, 64], [700]])
def test_whole_prompts(Hq, Hkv, D, lens):
    n = sum(lens)
    cu = tu.cumulative(lens)
    check(Hq, Hkv, D, draw(1, n, Hq, D), draw(2, n, Hkv, D), draw(3, n, Hkv, D), cu, None)


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 4, 64), (28, 4, 128), (16, 2, 128)])
@pytest.mark.parametrize("new,total", [([17], [400]), ([1, 1, 5], [129, 1, 128]), ([5, 9], [3, 0]), ([0, 4], [10, 4]), ([300], [290]), ([40, 100], [1000, 228])])
def test_prompts_that_continue_or_see_too_little(Hq, Hkv, D, new, total):
    check(Hq, Hkv, D, draw(4, sum(new), Hq, D), draw(5, sum(total), Hkv, D), draw(6, sum(total), Hkv, D), tu.cumulative(new), tu.cumulative(total))


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 4, 64), (28, 4, 128), (16, 1, 128), (5, 1, 64)])
@pytest.mark.parametrize("new,total", [([1], [5000]), ([40], [9000]), ([130, 1, 3, 0], [4100, 7000, 3, 900]), ([256, 17], [8192, 4113]), ([2, 2, 2, 2], [2500, 30, 2501, 1])])
def test_few_rows_over_many_keys(Hq, Hkv, D, new, total):
    """Tiles whose keys are cut over the chip, beside some that are not."""
    check(Hq, Hkv, D, draw(70, sum(new), Hq, D), draw(71, sum(total), Hkv, D), draw(72, sum(total), Hkv, D), tu.cumulative(new), tu.cumulative(total))


def test_many_sequences_some_over_many_keys():
    """More than 32 sequences of a few rows, the keys of some of them cut."""
    g = torch.Generator().manual_seed(76)
    new = torch.randint(0, 4, (45,), generator=g).tolist()
    total = [n + (5000 if i % 9 == 0 else 20 * i) for i, n in enumerate(new)]
    Hq, Hkv, D = 8, 1, 64
    check(Hq, Hkv, D, draw(77, sum(new), Hq, D), draw(78, sum(total), Hkv, D), draw(79, sum(total), Hkv, D), tu.cumulative(new), tu.cumulative(total))


def test_cut_keys_sharp_and_with_values_that_are_no_numbers():
    new, total, Hq, Hkv, D = [50], [6000], 14, 2, 128
    q, k, v = draw(73, 50, Hq, D, 8.0), draw(74, 6000, Hkv, D), draw(75, 6000, Hkv, D)
    cu_q, cu_k = tu.cumulative(new), tu.cumulative(total)
    clean, _ = check(Hq, Hkv, D, q, k, v, cu_q, cu_k)
    v[6000 - 20, 0, 5] = math.inf                            # row 29 is the last one that does not see it
    out, _ = tu.engine(Hq, Hkv, D).prompt(q, k, v, cu_q, cu_k)
    assert torch.equal(out[:30], clean[:30]) and torch.equal(out[:, 7:], clean[:, 7:])
    assert not torch.isfinite(out[30:, :7, 5]).any()
    others = [i for i in range(D) if i != 5]
    assert torch.equal(out[..., others], clean[..., others])


def test_no_keys_at_all():
    k = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = check(4, 2, 64, draw(7, 6, 4, 64), k, k, tu.cumulative([2, 4]), tu.cumulative([0, 0]))
    assert (out == 0).all() and (lse == -math.inf).all()


def test_many_short_sequences():
    g = torch.Generator().manual_seed(8)
    lens = torch.randint(0, 40, (333,), generator=g).tolist()
    n = sum(lens)
    check(8, 2, 128, draw(9, n, 8, 128), draw(10, n, 2, 128), draw(11, n, 2, 128), tu.cumulative(lens), None)


def test_rows_in_front_and_behind_stay():
    q, k, v = draw(12, 90, 4, 64), draw(13, 90, 2, 64), draw(14, 90, 2, 64)
    check(4, 2, 64, q, k, v, tu.cumulative([20, 31], first=7), tu.cumulative([20, 31], first=3))


@pytest.mark.parametrize("layout", ["fused", "head_major", "padded"])
def test_strides(layout):
    Hq, Hkv, D, lens = 16, 4, 64, [77, 5, 200]
    n = sum(lens)
    if layout == "fused":
        x = draw(15, n, Hq + 2 * Hkv, D)
        q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    elif layout == "head_major":
        q, k, v = (draw(16 + h, h, n, D).transpose(0, 1) for h in (Hq, Hkv, Hkv))
    else:
        q, k, v = (draw(20 + i, n, h, D + 24)[:, :, 8:8 + D] for i, h in enumerate((Hq, Hkv, Hkv)))
    check(Hq, Hkv, D, q, k, v, tu.cumulative(lens), None)


@pytest.mark.parametrize("size", [0.02, 6.0, 30.0])
def test_flat_and_sharp_softmax(size):
    """Rows whose weights are all alike, and rows of which one or two keys take all: the running maximum moves far."""
    lens = [513, 60]
    n = sum(lens)
    check(28, 4, 128, draw(23, n, 28, 128, size), draw(24, n, 4, 128), draw(25, n, 4, 128), tu.cumulative(lens), None)


def test_maximum_grows_along_the_keys():
    """Scores that rise with the key's position: every step of every row moves its maximum."""
    n, D = 900, 128
    q, k, v = draw(26, n, 4, D), draw(27, n, 1, D), draw(28, n, 1, D)
    q[..., 0] = 8.0
    k[..., 0] = (torch.arange(n, device="cuda").float()[:, None] / 8 - 50).to(torch.bfloat16)
    check(4, 1, D, q, k, v, tu.cumulative([n]), None)


@pytest.mark.parametrize("jump", [30.0, 60.0, 99.7, 100.0, 113.0, 125.7, 126.4, 127.9, 128.3, 400.0, 3000.0])
@pytest.mark.parametrize("D", [64, 128])
def test_one_key_far_above_the_first_ones(jump, D):
    """Scores that leave the range of the first keys' by 2^jump all at once, for some rows, some of them in one half of a step, one row
    twice."""
    n, Hq, Hkv = 700, 6, 2
    q, k, v = draw(60, n, Hq, D, 0.5), draw(61, n, Hkv, D, 0.5), draw(62, n, Hkv, D)
    q[..., 0] = torch.where(torch.arange(n, device="cuda")[:, None] % 3 == 0, 4.0, 0.0).to(torch.bfloat16)
    k[..., 0] = 0
    step = jump / (4.0 * D ** -0.5 * math.log2(math.e))
    for at, f in ((200, 1.0), (250, 1.01), (513, 2.0)):
        k[at, :, 0] = f * step
    check(Hq, Hkv, D, q, k, v, tu.cumulative([n]), None)


def test_softmax_scale():
    lens = [50, 129]
    n = sum(lens)
    check(4, 2, 64, draw(29, n, 4, 64), draw(30, n, 2, 64), draw(31, n, 2, 64), tu.cumulative(lens), None, softmax_scale=0.37)


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("D", [64, 128])
def test_what_a_row_does_not_see_does_not_reach_it(value, where, D):
    """A key or value that is no number: the rows in front of it, and every other sequence, are what they are without it."""
    lens, Hq, Hkv = [150, 77, 260], 14, 2
    n, bad = sum(lens), 150 + 40
    cu = tu.cumulative(lens)
    q, k, v = draw(32, n, Hq, D), draw(33, n, Hkv, D), draw(34, n, Hkv, D)
    eng = tu.engine(Hq, Hkv, D)
    clean, clean_lse = eng.prompt(q, k, v, cu, want_lse=True)
    (k if where == "k" else v)[bad, 0, 3] = value
    out, lse = eng.prompt(q, k, v, cu, want_lse=True)
    sees = torch.zeros(n, dtype=torch.bool, device="cuda")
    sees[bad:150 + 77] = True
    assert torch.equal(out[~sees], clean[~sees]) and torch.equal(lse[~sees], clean_lse[~sees])
    assert torch.equal(out[:, 7:], clean[:, 7:]) and torch.equal(lse[:, 7:], clean_lse[:, 7:])     # the other kv head
    if where == "v":                                       # it reaches its own coordinate of every row that sees it, and nothing else
        reached = out[sees][:, :7, 3].float()
        assert torch.isnan(reached).all() if math.isnan(value) else (reached == value).all()
        others = [i for i in range(D) if i != 3]
        assert torch.equal(out[sees][:, :7][..., others], clean[sees][:, :7][..., others]) and torch.equal(lse, clean_lse)
    elif math.isnan(value):
        assert torch.isnan(out[sees][:, :7]).all()


def test_large_head_count_and_long_rows():
    lens = [2000]
    check(64, 8, 64, draw(35, 2000, 64, 64), draw(36, 2000, 8, 64), draw(37, 2000, 8, 64), tu.cumulative(lens), None)


def test_nothing_but_empty_sequences():
    q, k, v = draw(80, 5, 4, 64), draw(81, 5, 2, 64), draw(82, 5, 2, 64)
    check(4, 2, 64, q, k, v, tu.cumulative([0, 0, 0], first=3), None)
    check(4, 2, 64, q, k, v, tu.cumulative([0]), tu.cumulative([5]))


def test_what_the_workspace_held_does_not_matter():
    q, k, v = draw(83, 20, 14, 128), draw(84, 4000, 2, 128), draw(85, 4000, 2, 128)
    eng, cu_q, cu_k = tu.engine(14, 2, 128), tu.cumulative([20]), tu.cumulative([4000])
    out, lse = eng.prompt(q, k, v, cu_q, cu_k, want_lse=True)
    eng._text_ws.fill_(255)
    again, lse2 = eng.prompt(q, k, v, cu_q, cu_k, want_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_bad_sequence_bounds_are_reported_and_not_followed():
    """Sequences that leave the tensors are not worked on; the others are."""
    q, k, v = draw(38, 64, 4, 64), draw(39, 64, 2, 64), draw(40, 64, 2, 64)
    eng = tu.engine(4, 2, 64)
    good, _ = eng.prompt(q, k, v, tu.cumulative([20, 44]))
    out = torch.full_like(good, 7.0)
    cu = torch.tensor([0, 20, 65], dtype=torch.int32, device="cuda")
    eng.prompt(q, k, v, cu, out=out)
    assert eng.text_status() == 1 and eng.text_status() == 0
    assert torch.equal(out[:20], good[:20]) and (out[20:] == 7).all()
    for cu in ([0, -3, 64], [0, 40, 20], [-5, 20, 64]):
        eng.prompt(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), out=out)
        assert eng.text_status() == 1


def test_captured_call_follows_its_inputs():
    lens, Hq, Hkv, D = [100, 60], 8, 2, 128
    n = sum(lens)
    q, k, v, cu = draw(41, n, Hq, D), draw(42, n, Hkv, D), draw(43, n, Hkv, D), tu.cumulative(lens)
    eng = tu.engine(Hq, Hkv, D)
    out, lse = eng.prompt(q, k, v, cu, want_lse=True)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        eng.prompt(q, k, v, cu, out=out, lse=lse)
    q.copy_(draw(44, n, Hq, D))
    cu.copy_(tu.cumulative([10, 150]))
    for _ in range(3):
        out.zero_()
        g.replay()
    mine, want, want_lse, tol, ltol = tu.prompt_reference(q, k, v, cu, cu, D ** -0.5)
    tu.assert_close(out, want, tol, "out")
    tu.assert_lse(lse, want_lse, ltol)


def test_same_result_every_time_and_on_another_stream():
    lens = [33, 500, 260]
    n = sum(lens)
    q, k, v, cu = draw(45, n, 28, 128), draw(46, n, 4, 128), draw(47, n, 4, 128), tu.cumulative(lens)
    eng = tu.engine(28, 4, 128)
    first, lse = eng.prompt(q, k, v, cu, want_lse=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        with torch.cuda.stream(s):
            again, lse2 = eng.prompt(q, k, v, cu, want_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(first, again) and torch.equal(lse, lse2)


def test_refusals():
    eng = tu.engine(4, 2, 64)
    q, k, v, cu = draw(48, 8, 4, 64), draw(49, 8, 2, 64), draw(50, 8, 2, 64), tu.cumulative([8])
    for bad in [(q.half(), k, v, cu), (q, k[:, :1], v, cu), (q.cpu(), k, v, cu), (q, k, v[:5], cu), (q, k, v, cu.long()), (q.transpose(1, 2), k, v, cu), (q, k, v, cu.cpu())]:
        with pytest.raises(binding.AdasparkError):
            eng.prompt(*bad)
    for bad in [(q[:1].expand(8, 4, 64), k, v, cu), (q, k[:, :1].expand(8, 2, 64), v, cu), (q, k, v, cu.view(1, 2)), (q, k, v, cu[:0])]:
        with pytest.raises(binding.AdasparkError):
            eng.prompt(*bad)
    for kw in [dict(out=torch.empty_like(q)[:4]), dict(out=torch.empty_like(q).float()), dict(lse=torch.empty(8, 4, dtype=torch.float64, device="cuda"))]:
        with pytest.raises(binding.AdasparkError):
            eng.prompt(q, k, v, cu, **kw)
