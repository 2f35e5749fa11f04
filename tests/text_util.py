"""Plain 64-bit forms of the text operators (packed causal attention, the 8-bit rows of the paged cache), and the bounds that
their outputs are held to."""
import math

import torch

from paper_2604_08077_b200 import binding

BF16_HALF = 2.0 ** -8          # the most that rounding to bf16 moves a value, relative to it (torch.finfo(torch.bfloat16).eps / 2)


def engine(Hq, Hkv, D, **kw):
    return binding.AdaSAttn(cube=(4, 4, 4), n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, top_p=0.9, **kw)


def cumulative(lens, first=0):
    c = [first]
    for n in lens:
        c.append(c[-1] + n)
    return torch.tensor(c, dtype=torch.int32, device="cuda")


def attend(q, k, v, last, scale):
    """Rows q [r, Hq, D] over k, v [n, Hkv, D] in 64 bits, row i seeing the keys 0 .. last[i].  Returns (out, lse, out_tol, lse_tol).

    The bounds.  A score is a sum of D products in 32 bits, off by at most (D + 8) 2^-23 of the sum of their magnitudes: `ds`, in units of
    the exponent; its scale and reference round again, 2^-22 of the score's magnitude.  A weight is then off by that, by 2^-17 for
    the exponential itself, and by 2^-8 of itself where it is rounded to bf16 for the product with V; the 32-bit sums of n weights and
    products add 2^-22 sqrt(n) at most here.  Weight errors e move an output by at most 2 e sum(w |v|) (numerator and denominator).  The
    output's own rounding is 2^-8 of it."""
    D, G = q.shape[-1], q.shape[1] // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    hidden = torch.arange(k.shape[0], device=q.device)[None, :] > last[:, None]
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    tol, ltol = torch.zeros_like(q), torch.zeros_like(lse)
    for h in range(q.shape[1]):
        kk, vv = k[:, h // G], v[:, h // G]
        logits = (q[:, h] @ kk.T * scale).masked_fill(hidden, -math.inf)
        if k.shape[0]:
            mags = (q[:, h].abs() @ kk.abs().T * scale).masked_fill(hidden, 0).amax(1)
            lse[:, h] = torch.logsumexp(logits, 1)
        else:
            mags = torch.zeros(q.shape[0], dtype=torch.float64, device=q.device)
        w = torch.exp(logits - torch.where(lse[:, h] == -math.inf, 0.0, lse[:, h])[:, None])
        w = torch.where(hidden, 0.0, w)
        # (values that no row may see take no part: 0 times an infinity would be one)
        out[:, h] = w @ torch.where(hidden.all(0)[:, None], 0.0, vv)
        size = w @ torch.where(hidden.all(0)[:, None], 0.0, vv).abs()
        e = ((D + 8) * 2.0 ** -23 + 2.0 ** -22) * mags + 2.0 ** -17 + 2.0 ** -22 * math.sqrt(max(1, k.shape[0]))
        ltol[:, h] = e + 2.0 ** -22 * lse[:, h].abs().nan_to_num(posinf=0.0)
        tol[:, h] = BF16_HALF * out[:, h].abs() + (BF16_HALF + 2 * e)[:, None] * size + 1e-30
    return out, lse, tol, ltol


def prompt_reference(q, k, v, cu_q, cu_k, scale):
    """attend() for packed sequences; rows of no sequence are None in the mask that comes first."""
    cq, ck = cu_q.tolist(), cu_k.tolist()
    n_q, Hq, D = q.shape
    mine = torch.zeros(n_q, dtype=torch.bool, device=q.device)
    got = [torch.zeros(n_q, Hq, D, dtype=torch.float64, device=q.device), torch.zeros(n_q, Hq, dtype=torch.float64, device=q.device),
           torch.zeros(n_q, Hq, D, dtype=torch.float64, device=q.device), torch.zeros(n_q, Hq, dtype=torch.float64, device=q.device)]
    for b in range(len(cq) - 1):
        rows, keys = slice(cq[b], cq[b + 1]), slice(ck[b], ck[b + 1])
        n, m = cq[b + 1] - cq[b], ck[b + 1] - ck[b]
        if n == 0:
            continue
        mine[rows] = True
        last = torch.arange(n, device=q.device) + (m - n)
        for t, x in zip(got, attend(q[rows], k[keys], v[keys], last, scale)):
            t[rows] = x
    return mine, *got


def assert_close(got, want, tol, what):
    assert got.shape == want.shape
    if got.numel() == 0:
        return
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got.double() - want).abs() - tol
    worst = over.argmax()
    assert over.max() <= 0, f"{what}: off by {(got.double() - want).abs().flatten()[worst]:.3e}, bound {tol.flatten()[worst]:.3e}, {int((over > 0).sum())} of {over.numel()}"


def assert_lse(got, want, tol, what="lse"):
    empty = want == -math.inf
    assert torch.equal(got == -math.inf, empty), f"{what}: rows that see nothing"
    assert_close(got[~empty], want[~empty], tol[~empty], what)


def quantise(x):
    """What an e4m3 page holds of rows x [..., D], by the definition, in 64 bits: (values, byte of the power of two)."""
    x = x.double()
    finite = torch.isfinite(x)
    top = torch.where(finite, x.abs(), 0.0).amax(-1, keepdim=True)
    byte = torch.zeros_like(top)
    for s in range(248):                                         # the smallest s with top <= 448 * 2^(s - 127)
        byte = torch.where((byte == s) & (top > 448.0 * 2.0 ** (s - 127)), s + 1.0, byte)
    y = x / torch.exp2(byte - 127)
    a = torch.where(finite, y.abs(), 1.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)      # exact: a is a bf16 number times a power of two
    y = torch.where(finite, torch.round(y / step) * step, math.nan)
    return y * torch.exp2(byte - 127), byte[..., 0].to(torch.uint8)


def page_values(cache):
    """The values that a cache's pages stand for, in 64 bits: two tensors [pages, heads, page size, D]."""
    got = []
    for p, s in ((cache.k_pages, cache.k_scale), (cache.v_pages, cache.v_scale)):
        x = p.to(torch.float32).double()
        got.append(x if s is None else x * torch.exp2(s.double() - 127)[..., None])
    return got


def sequence_values(cache, table, b, n):
    """Keys and values of the first n tokens of sequence b in 64 bits: [n, heads, D]."""
    page = cache.page_size
    cols = table[b, :-(-n // page)].long()
    return [x[cols].permute(0, 2, 1, 3).reshape(-1, cache.n_kv_heads, cache.head_dim)[:n] for x in page_values(cache)]


def scattered(g, per_sequence, n_spare=2):
    """A block table whose pages lie in no order, and the number of pages of its pool."""
    total = sum(per_sequence) + n_spare
    order = torch.randperm(total, generator=g).to(torch.int32)
    table = torch.full((len(per_sequence), max(1, max(per_sequence))), -7, dtype=torch.int32)   # columns that nothing may read
    at = 0
    for i, n in enumerate(per_sequence):
        table[i, :n] = order[at:at + n]
        at += n
    return table.cuda(), total
