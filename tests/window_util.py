"""64-bit forms of rotated rows and of attention by a window over a paged cache, and the bounds that outputs are held to."""
import math

import torch

from text_util import BF16_HALF


def hidden_from(first, rows, n, window, sinks, device="cuda"):
    """[rows, n]: which of the positions 0 .. n - 1 the tokens first .. first + rows - 1 do not see."""
    p, j = torch.arange(first, first + rows, device=device)[:, None], torch.arange(n, device=device)[None, :]
    sees = j <= p
    if window:
        sees &= (j > p - window) | (j < sinks)
    return ~sees


def attend_masked(q, k, v, hidden, scale):
    """Rows q [r, Hq, D] over k, v [n, Hkv, D] in 64 bits.  Returns (out, lse, out_tol, lse_tol); what a row does not see does not reach it.

    The bounds.  A score is a sum of D products in 32 bits, off by at most (D + 8) 2^-23 of the sum of their magnitudes, in units of the
    exponent; its scale and reference round again, 2^-22 of its magnitude.  A weight is off by that, by 2^-17 for the exponential, and by 2^-8
    of itself where it is rounded to bf16 for the product with V; 32-bit sums of n weights add 2^-22 sqrt(n).  Weight errors e move an output
    by at most 2 e sum(w |v|).  The output's own rounding is 2^-8 of it."""
    D, G = q.shape[-1], q.shape[1] // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    tol, ltol = torch.zeros_like(q), torch.zeros_like(lse)
    if k.shape[0] == 0:
        return out, lse, tol + 1e-30, ltol
    gone = hidden.all(0)[:, None]
    for h in range(q.shape[1]):
        kk, vv = torch.where(gone, 0.0, k[:, h // G]), torch.where(gone, 0.0, v[:, h // G])
        logits = (q[:, h] @ kk.T * scale).masked_fill(hidden, -math.inf)
        mags = (q[:, h].abs() @ kk.abs().T * scale).masked_fill(hidden, 0).amax(1)
        lse[:, h] = torch.logsumexp(logits, 1)
        w = torch.exp(logits - torch.where(lse[:, h] == -math.inf, 0.0, lse[:, h])[:, None]).masked_fill(hidden, 0)
        out[:, h] = w @ vv
        size = w @ vv.abs()
        e = ((D + 8) * 2.0 ** -23 + 2.0 ** -22) * mags + 2.0 ** -17 + 2.0 ** -22 * math.sqrt(k.shape[0])
        ltol[:, h] = e + 2.0 ** -22 * lse[:, h].abs().nan_to_num(posinf=0.0)
        tol[:, h] = BF16_HALF * out[:, h].abs() + (BF16_HALF + 2 * e)[:, None] * size + 1e-30
    return out, lse, tol, ltol


def chunk_reference(q, cu, kv_len, sequence, window, sinks, scale):
    """attend_masked for packed rows over a cache; sequence(b, n) gives its keys and values [n, Hkv, D].  Returns (rows of some sequence, ...)."""
    n_q, Hq, D = q.shape
    mine = torch.zeros(n_q, dtype=torch.bool, device=q.device)
    got = [torch.zeros(n_q, Hq, D, dtype=torch.float64, device=q.device), torch.zeros(n_q, Hq, dtype=torch.float64, device=q.device),
           torch.zeros(n_q, Hq, D, dtype=torch.float64, device=q.device), torch.zeros(n_q, Hq, dtype=torch.float64, device=q.device)]
    for b, n in enumerate(kv_len):
        r = cu[b + 1] - cu[b]
        if r == 0:
            continue
        rows = slice(cu[b], cu[b + 1])
        mine[rows] = True
        k, v = sequence(b, n)
        hidden = hidden_from(n - r, r, n, window, sinks, q.device)
        for t, x in zip(got, attend_masked(q[rows], k, v, hidden, scale)):
            t[rows] = x
    return mine, *got


def rotated(x, weight, positions, frequencies, axis, adjacent, eps):
    """Rows x [n, heads, D] with their norm and rotation in 64 bits, and the bound of a 32-bit evaluation before its rounding.

    The bound.  Squares and their sum are off by (D + 2) 2^-24 of it, half of which reaches its root; 1/sqrt by 2^-22; an angle by 2^-24 of
    half a turn (as a 32-bit number of half turns), its cosine and sine by 2^-22 more; four products and sums round by 2^-24 each: 2^-16 of |a| + |b|
    is more than all of them for D up to 128."""
    x = x.double()
    D = x.shape[-1]
    if weight is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * weight.double()
    y, size = x.clone(), x.abs()
    pairs = len(frequencies)
    if pairs:
        p = positions.reshape(-1, x.shape[0]).double()
        f = torch.tensor(frequencies, dtype=torch.float64, device=x.device)
        t = p[torch.tensor(axis, device=x.device)].T * f
        c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
        first = slice(0, 2 * pairs, 2) if adjacent else slice(0, pairs)
        second = slice(1, 2 * pairs, 2) if adjacent else slice(pairs, 2 * pairs)
        a, b = x[..., first], x[..., second]
        y[..., first], y[..., second] = a * c - b * s, b * c + a * s
        size[..., first] = size[..., second] = a.abs() + b.abs()
    assert D <= 128
    return y, size * 2.0 ** -16
