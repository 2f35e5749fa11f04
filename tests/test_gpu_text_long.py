"""GPU test of a decode step over the longest sequence that a block table has room for."""
import math

import pytest
import torch

import text_util as tu
from paper_2604_08077_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_over_nearly_2_31_tokens(e4m3):
    """One page of 16 tokens, listed 2^27 - 1 times.  The query is zero, so every weight is 1: numbers of tokens and sums of a few powers of
    two are exact in 32 bits up to the join of some hundred parts."""
    D, page, width = 64, 16, (1 << 27) - 1
    n = page * width
    row = torch.tensor([1.0, 0.5, -2.0, 0.0], device="cuda").repeat(D // 4)
    k = torch.randn(1, 1, page, D, generator=torch.Generator().manual_seed(230)).cuda()
    dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    scales = [torch.full((1, 1, page), 127, dtype=torch.uint8, device="cuda") for _ in range(2)] if e4m3 else []
    cache = binding.PagedCache(k.to(dtype), row.expand(1, 1, page, D).to(dtype).contiguous(), *scales)
    table, kv_len = torch.zeros(2, width, dtype=torch.int32, device="cuda"), torch.tensor([n, 5], dtype=torch.int32, device="cuda")
    eng = tu.engine(2, 1, D)
    out, lse = eng.paged_decode(torch.zeros(2, 2, D, dtype=torch.bfloat16, device="cuda"), None, None, cache, table, kv_len, want_lse=True)
    assert eng.text_status() == 0
    assert torch.equal(out.float(), row.expand(2, 2, D))
    want = torch.tensor([math.log(n), math.log(5)], device="cuda")[:, None]
    # the logarithm in 32 bits (2^-23 of it), and 296 parts' sums rounded as they are added (2^-24 each at most)
    assert ((lse - want).abs() <= want * 2.0 ** -22 + 296 * 2.0 ** -24).all()


def test_a_million_sequences_beside_a_long_prompt():
    """What is planned between two tiles of a CTA takes more than 2 s here: 147 levels of 10^6 sequences."""
    D, B, long = 64, 1_000_000, 40_000
    at = B // 3
    lens = torch.ones(B, dtype=torch.int64)
    lens[at] = long
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)]).to(torch.int32).cuda()
    n = int(lens.sum())
    g = torch.Generator(device="cuda").manual_seed(231)
    q, k, v = (torch.randn(n, 1, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    eng = tu.engine(1, 1, D)
    out, lse = eng.prompt(q, k, v, cu, want_lse=True)
    assert eng.text_status() == 0
    one = torch.ones(n, dtype=torch.bool, device="cuda")
    one[at:at + long] = False
    assert torch.equal(out[one], v[one])                             # a weight of 1
    rows = torch.tensor([0, 1, 127, 5000, 20_001, 39_872, 39_999], device="cuda")
    kk, vv = k[at:at + long], v[at:at + long]
    want, wl, tol, ltol = tu.attend(q[at + rows], kk, vv, rows, D ** -0.5)
    tu.assert_close(out[at + rows], want, tol, "out")
    tu.assert_lse(lse[at + rows], wl, ltol)
