"""Norms of rows whose squares leave 32 bits at either end, with an eps of zero, tiny or large, against 64 bits."""
import pytest
import torch

from test_gpu_rotary import check, rand, turn
from text_util import engine, page_values, scattered
from window_util import rotated

pytestmark = pytest.mark.gpu

# magnitudes of the rows, as powers of two; -133 is the smallest bf16 number
POWERS = [-133, -126, -120, -100, -80, -75, -70, -63, -56, -51, -50, -49, -30, 0, 30, 58, 59, 60, 63, 80, 120]


def rows_of(g, heads, D, least=-1):
    """A token a magnitude (or a bit more), heads of normal draws of it; the smallest: a multiple of the smallest number."""
    x = torch.randn(len(POWERS), heads, D, generator=g, dtype=torch.float64).clamp(-4, 4)
    x = x * torch.exp2(torch.tensor(POWERS, dtype=torch.float64))[:, None, None]
    x[0] = torch.randint(least, 3, (heads, D), generator=g).double() * 2.0 ** -133
    return x.to(torch.bfloat16).cuda()


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -149, 2.0 ** -130, 2.0 ** -101, 2.0 ** -100, 2.0 ** -20, 2.0 ** 100, 2.0 ** 118, 2.0 ** 127, 3.4028234663852886e38])
@pytest.mark.parametrize("Hq,Hkv,D,adjacent", [(28, 4, 128, False), (4, 2, 64, True)])
def test_rows_of_any_magnitude(Hq, Hkv, D, adjacent, eps):
    g = torch.Generator().manual_seed(17)
    eng = engine(Hq, Hkv, D)
    r, freq, axis = turn(D, [D // 4], adjacent)
    q, k, wq, wk = rows_of(g, Hq, D), rows_of(g, Hkv, D), rand(g, D), rand(g, D)
    pos = torch.randint(0, 5000, (q.shape[0],), generator=g, dtype=torch.int32).cuda()
    qo, ko = eng.rotate(q, k, pos, r, q_norm=wq, k_norm=wk, eps=eps)
    # (a large eps makes outputs that bf16 holds as subnormal numbers: steps of 2^-133; a row times a power of two may lose what lies below 2^-149 of 32 bits, times the root's inverse)
    for got, x, w, what in ((qo, q, wq, "q"), (ko, k, wk, "k")):
        want, tol = rotated(x, w, pos, freq, axis, adjacent, eps)
        tol = tol + 2.0 ** -8 * want.abs() + 2.0 ** -133
        assert torch.isfinite(got).all(), what
        over = (got.double() - want).abs() - tol
        assert over.max() <= 0, (what, [POWERS[i] for i in (over.flatten(1).amax(1) > 0).nonzero().flatten().tolist()])


@pytest.mark.parametrize("D", [64, 128])
def test_a_row_of_zeros_without_eps_holds_no_numbers(D):
    """0 / sqrt(0), as the formula has it; its neighbours in the same warps stay."""
    g = torch.Generator().manual_seed(18)
    eng = engine(8, 2, D)
    q, w = rand(g, 9, 8, D), rand(g, D)
    q[4, 3] = 0
    qo, _ = eng.rotate(q, None, q_norm=w, eps=0.0)
    assert qo[4, 3].isnan().all()
    q[4, 3], qo[4, 3] = 1, w
    check(qo, q, w, torch.zeros(9, dtype=torch.int32, device="cuda"), [], [], False, "q", eps=0.0)
    q[4, 3] = 0
    qo, _ = eng.rotate(q, None, q_norm=w, eps=1e-30)
    assert (qo[4, 3] == 0).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_such_keys_into_pages(e4m3):
    g = torch.Generator().manual_seed(19)
    Hq, Hkv, D, page = 4, 2, 128, 16
    eng = engine(Hq, Hkv, D)
    r, freq, axis = turn(D, [64], False)
    k, w = rows_of(g, Hkv, D), rand(g, D)
    n = k.shape[0]
    table, n_pages = scattered(g, [-(-n // page)])
    cache = eng.paged_cache(n_pages, page, e4m3=e4m3)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    eng.paged_append(cache, None, k, k, ints([0, n]), table, ints([n]), r, k_norm=w, eps=0.0)
    assert eng.text_status() == 0
    at = torch.arange(n, device="cuda")
    got = page_values(cache)[0][table[0].long()[at // page], :, at % page]
    want, tol = rotated(k, w, at, freq, axis, False, 0.0)
    # a code is off by half a step of 2^-3 of a value, or of the smallest step of its row: 2^-9 times its power of two, the row's largest being above 2^7.8 of that
    own = want.abs() * 2.0 ** -4 + want.abs().amax(-1, keepdim=True) * 2.0 ** -17 if e4m3 else want.abs() * 2.0 ** -8
    assert torch.isfinite(got).all() and ((got - want).abs() <= 1.1 * tol + own + 1e-30).all()
