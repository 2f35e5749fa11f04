"""Chunks over pages among very many sequences: no tile under way waits for the next one to be planned."""
import pytest
import torch

from paper_2604_08077_b200 import binding
from test_gpu_paged_prompt import ints, rand
from text_util import assert_close, assert_lse, engine, sequence_values
from window_util import attend_masked, hidden_from

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_million_sequences_beside_a_long_chunk(e4m3):
    """What is planned between two tiles of a pair takes more than 2 s here: 150 levels of 10^6 sequences, of which all but one are a token that sees itself
    (they may share a page: nobody writes)."""
    D, B, long, page = 64, 1_000_000, 40_000, 256
    at, width = B // 3, -(-40_000 // 256)
    g = torch.Generator().manual_seed(232)
    n_pages = width + 5
    k, v = rand(g, n_pages, 1, page, D), rand(g, n_pages, 1, page, D)
    if e4m3:
        codes = [x.float().mul(16).to(torch.float8_e4m3fn) for x in (k, v)]
        cache = binding.PagedCache(*codes, *(torch.full(k.shape[:3], 123, dtype=torch.uint8, device="cuda") for _ in range(2)))
    else:
        cache = binding.PagedCache(k, v)
    table = torch.full((B, width), -3, dtype=torch.int32, device="cuda")
    table[:, 0] = width + torch.arange(B, device="cuda") % 5
    table[at] = torch.randperm(width, generator=g).to(torch.int32).cuda()
    lens = torch.ones(B, dtype=torch.int32, device="cuda")
    lens[at] = long
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), lens.long().cumsum(0)]).to(torch.int32)
    n = int(cu[-1])
    q = rand(g, n, 1, D)
    eng = engine(1, 1, D)
    out, lse = eng.paged_prompt(q, cache, cu, table, lens, want_lse=True)
    assert eng.text_status() == 0
    keys, values = sequence_values(cache, table, at, long)
    first = torch.stack([sequence_values(cache, table, b, 1)[1][0] for b in range(5)])     # a weight of 1
    for a, b in ((0, at), (at + 1, B)):
        rows = slice(a if a == 0 else a + long - 1, b if a == 0 else b + long - 1)
        assert torch.equal(out[rows], first[torch.arange(a, b, device="cuda") % 5].to(torch.bfloat16))
    for r in (0, 1, 127, 5000, 20_001, 39_872, 39_999):
        row = slice(at + r, at + r + 1)
        want, wl, tol, ltol = attend_masked(q[row], keys[:r + 1], values[:r + 1], hidden_from(r, 1, r + 1, 0, 0), D ** -0.5)
        if e4m3:                                                 # q in two parts: 2^-18 of its largest magnitude, as a score
            e = q[row].double().abs().amax(-1) * 2.0 ** -18 * keys.abs().sum(-1).amax() * D ** -0.5
            tol, ltol = tol + (2 * e * values.abs().amax())[..., None], ltol + e
        assert_close(out[row], want, tol, f"row {r}")
        assert_lse(lse[row], wl, ltol)
