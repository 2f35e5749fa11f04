"""The operators for text beside the video: what a program that serves requests without a video, or the text turns
that follow one, has this library do, as a set of measurable cases.

Three operators that work on the same packed sequences and the same paged cache:

  prompt  causal softmax attention over whole prompts, sequences of different lengths packed one behind the other
          (token i of a sequence of n_q new and n_k present tokens sees the tokens 0 .. n_k - n_q + i), grouped heads,
          with the logarithm of each row's sum
  cache   new keys and values written into the pages of a cache, as bf16 or as 8-bit floats with a power of two per
          token and head, and read back
  decode  attention of one new token per sequence over the pages of its cache

8-bit pages: a row x of head_dim values is held as e4m3 codes c and one byte s, x ~ c * 2^(s - 127), with the smallest
power of two for which the row's largest magnitude is at most 448 (s in 0 .. 247).
"""
from __future__ import annotations

import math

import torch

own = False

_BASE = {
    "kind": "prompt", "lens": "41", "ctx": "", "Hq": 28, "Hkv": 4, "D": 128, "fused": True,   # prompt
    "page": 16, "e4m3": False, "append": False,                                               # cache, decode
}


def _case(name, **kw):
    return {**_BASE, **kw, "name": name}


def listed():
    return [
        # One short question of a single user: nothing but latency.
        _case("prompt_question", lens="41"),
        # What a scheduler packs into one step: short and ordinary prompts, a single token among them.
        _case("prompt_batch_mixed", lens="512,1,37,1024,129,2048,7,300"),
        # The smaller heads, queries and keys in tensors of their own.
        _case("prompt_d64", lens="1,700,64,1536,2000", Hq=16, Hkv=4, D=64, fused=False),
        # New turns of conversations whose earlier tokens are read back from a cache.
        _case("prompt_continued", lens="256,17,64,1", ctx="7936,4096,0,1023", fused=False),
        # Two long documents.
        _case("prompt_long", lens="8192,8192"),
        # One decode step's keys and values of sixteen sequences, read back: latency.
        _case("cache_step", kind="cache", lens="1x16", ctx="1000x16"),
        # Ordinary prompts of odd lengths into 8-bit pages, small heads.
        _case("cache_prompts_e4m3_d64", kind="cache", lens="700,1,2049,333,64,1535", ctx="0,15,100,0,64,0", Hq=16, Hkv=4, D=64, e4m3=True),
        # The tokens of the longest video of the benchmark, kept in 8 bits.
        _case("cache_128k_e4m3", kind="cache", lens="131072", page=64, e4m3=True),
        # One conversation, one new token: latency.
        _case("decode_single", kind="decode", lens="544", append=True),
        # One conversation about a very long document: the cache's length is all there is to share out.
        _case("decode_128k_single_e4m3", kind="decode", lens="131072", page=64, e4m3=True),
        # Serving: a batch of conversations of any length, one slot of the batch unused.
        _case("decode_batch_ragged", kind="decode", append=True,
              lens="5000,1,17,8192,300,0,4097,2500,64,1023,777,6000,128,129,3333,50,2048,1500,900,7000,15,16,450,5555"),
        # Serving: sixteen conversations of the longest length, in 8 bits.
        _case("decode_128k_b16_e4m3", kind="decode", lens="131584x16", page=64, e4m3=True),
    ]


_HEADS = [(4, 4, 64), (16, 4, 64), (8, 2, 128), (16, 2, 128), (28, 4, 128), (28, 4, 128)]
_MAX_PAIRS = 28 * 8192 * 8192            # (query head, row, key) triples of the largest prompt case
_MAX_CACHE_TOKENS = 16 * 131584 * 4 * 128   # tokens * kv heads * head_dim of the largest decode case
_MAX_WRITE_TOKENS = 131072 * 4 * 128


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["prompt", "prompt", "cache", "decode", "decode"])
        Hq, Hkv, D = rng.choice(_HEADS)
        c = {**_BASE, "kind": kind, "Hq": Hq, "Hkv": Hkv, "D": D, "fused": rng.random() < 0.5,
             "page": rng.choice([16, 16, 32, 64, 128]), "e4m3": rng.random() < 0.5}
        n = _log_uniform(rng, 1, 24)
        top = _log_uniform(rng, 16, {"prompt": 8192, "cache": 65536, "decode": 131072}[kind])
        lens = [max(1, _log_uniform(rng, max(1, top // 16), top)) for _ in range(n)]
        ctx = [0] * n
        if kind != "decode" and rng.random() < 0.4:
            ctx = [rng.choice([0, _log_uniform(rng, 1, 4096)]) for _ in range(n)]
        if kind == "prompt":
            c.update(e4m3=False, page=16, fused=c["fused"] and not any(ctx))
            if sum(Hq * a * (a + 2 * b) for a, b in zip(lens, ctx)) > _MAX_PAIRS or n * Hq * max(lens) * (max(lens) + max(ctx)) > 2 * _MAX_PAIRS:
                continue
        elif kind == "cache":
            c.update(fused=True)
            if sum(lens) * Hkv * D > _MAX_WRITE_TOKENS:
                continue
        else:
            c.update(fused=True, append=not c["e4m3"] and rng.random() < 0.5)
            if n > 1 and rng.random() < 0.3:
                lens[rng.randrange(n)] = 0
            if n * max(lens) * Hkv * D * (1 if c["e4m3"] else 2) > _MAX_CACHE_TOKENS:
                continue
        c["lens"] = ",".join(map(str, lens))
        c["ctx"] = ",".join(map(str, ctx)) if any(ctx) else ""
        return c


def _numbers(text):
    got = []
    for part in text.split(",") if text else []:
        value, _, times = part.partition("x")
        got += [int(value)] * int(times or 1)
    return got


def _lens(case):
    """(new tokens, tokens before them) of each sequence."""
    new = _numbers(case["lens"])
    return new, _numbers(case["ctx"]) or [0] * len(new)


# ---------------------------------------------------------------------------------------------------------------- inputs

def _cumulative(lens, device):
    c = [0]
    for n in lens:
        c.append(c[-1] + n)
    return torch.tensor(c, dtype=torch.int32, device=device)


def _quantise(x):
    """[..., D] values -> e4m3 codes and the byte of the row's power of two."""
    x = x.float()
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)                                   # top = m * 2^e, m in [0.5, 1)
    s = (e - 9 + (m > 0.875) + 127).clamp(0, 247)             # 448 = 0.875 * 2^9
    s = torch.where(top == 0, torch.zeros_like(s), s)
    return torch.ldexp(x, (127 - s)[..., None]).to(torch.float8_e4m3fn), s.to(torch.uint8)


def _values(codes, s):
    return codes.float() * torch.ldexp(torch.ones_like(s, dtype=torch.float32), s.to(torch.int32) - 127)[..., None]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    Hq, Hkv, D, page = case["Hq"], case["Hkv"], case["D"], case["page"]
    new, ctx = _lens(case)
    total = [a + b for a, b in zip(new, ctx)]
    randn = lambda *s: torch.randn(*s, generator=g, device=dev).to(torch.bfloat16)  # noqa: E731
    st = {"case": dict(case), "kind": case["kind"], "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "scale": D ** -0.5, "max_total": max(total)}
    if case["kind"] == "prompt":
        n_q, n_k = sum(new), sum(total)
        if case["fused"]:                                     # slices of what one projection gives
            qkv = randn(n_q, Hq + 2 * Hkv, D)
            st["q"], st["k"], st["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        else:
            st["q"], st["k"], st["v"] = randn(n_q, Hq, D), randn(n_k, Hkv, D), randn(n_k, Hkv, D)
        st["cu_q"], st["cu_k"], st["max_new"] = _cumulative(new, dev), _cumulative(total, dev), max(new)
        st["out"] = torch.empty(n_q, Hq, D, dtype=torch.bfloat16, device=dev)
        st["lse"] = torch.empty(n_q, Hq, dtype=torch.float32, device=dev)
    else:
        # a pool of pages in no order, the sequences' pages scattered over it
        per = [-(-n // page) for n in total]
        n_pages, width = sum(per) + 3, max(per)
        order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
        table = torch.zeros(len(per), width, dtype=torch.int32, device=dev)
        at = 0
        for i, n in enumerate(per):
            table[i, :n] = order[at:at + n]
            at += n
        st["table"], st["kv_len"] = table, torch.tensor(total, dtype=torch.int32, device=dev)
        k, v = randn(n_pages, Hkv, page, D), randn(n_pages, Hkv, page, D)
        if case["e4m3"]:
            (st["k_pages"], st["k_scale"]), (st["v_pages"], st["v_scale"]) = _quantise(k), _quantise(v)
        else:
            st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"] = k, v, None, None
        if case["kind"] == "cache":
            n = sum(new)
            if case["fused"]:
                kv = randn(n, 2 * Hkv, D)
                st["k"], st["v"] = kv[:, :Hkv], kv[:, Hkv:]
            else:
                st["k"], st["v"] = randn(n, Hkv, D), randn(n, Hkv, D)
            # the rows differ in size, as keys behind a norm and values do
            grow = torch.exp2(torch.randint(-6, 7, (n, 1, 1), generator=g, device=dev).float()).to(torch.bfloat16)
            st["k"].mul_(grow), st["v"].mul_(grow)
            st["cu"], st["max_new"] = _cumulative(new, dev), max(new)
            st["k_out"], st["v_out"] = torch.empty(n, Hkv, D, dtype=torch.bfloat16, device=dev), torch.empty(n, Hkv, D, dtype=torch.bfloat16, device=dev)
        else:
            B = len(new)
            st["q"] = randn(B, Hq, D)
            st["k"], st["v"] = (randn(B, Hkv, D), randn(B, Hkv, D)) if case["append"] else (None, None)
            st["live"] = torch.tensor([i for i, n in enumerate(total) if n], device=dev)
            st["out"] = torch.empty(B, Hq, D, dtype=torch.bfloat16, device=dev)
            st["lse"] = torch.empty(B, Hq, dtype=torch.float32, device=dev)
    if own:
        from paper_2604_08077_b200 import binding
        st["eng"] = binding.AdaSAttn(cube=(4, 4, 4), n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, top_p=0.9)
        if case["kind"] != "prompt":
            st["cache"] = binding.PagedCache(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
    return st


# ---------------------------------------------------------------------------------------------------------------- plain forms

def _attend(q, k, v, visible, scale):
    """q [B, h, r, d], k and v [B, h, n, d] in 32 bits, visible [B, 1, r, n]: outputs and the logarithms of the sums."""
    s = torch.matmul(q * scale, k.transpose(-1, -2))
    s.masked_fill_(~visible, -math.inf)
    m = s.amax(-1, keepdim=True)
    s.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    l = s.sum(-1, keepdim=True)
    o = torch.matmul(s, v) / torch.where(l > 0, l, torch.ones_like(l))
    return o, (m + torch.log(l))[..., 0]


def _plain_prompt(st):
    q, k, v, cu_q, cu_k = st["q"], st["k"], st["v"], st["cu_q"].long(), st["cu_k"].long()
    B, Hq, Hkv, D, dev = cu_q.numel() - 1, st["Hq"], st["Hkv"], st["D"], q.device
    G, Lq, Lk = Hq // Hkv, st["max_new"], st["max_total"]
    rq, rk = torch.arange(Lq, device=dev), torch.arange(Lk, device=dev)
    n_q, n_k = cu_q.diff(), cu_k.diff()
    iq = (cu_q[:-1, None] + rq).clamp(max=q.shape[0] - 1)
    ik = (cu_k[:-1, None] + rk).clamp(max=k.shape[0] - 1)
    last = n_k[:, None] - n_q[:, None] + rq                                            # the last key that a row sees
    visible = (rk <= last[:, :, None])[:, None, None].expand(B, 1, G, Lq, Lk).reshape(B, 1, G * Lq, Lk)
    qs = q[iq].float().view(B, Lq, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Lq, D)
    ks, vs = (x[ik].float().permute(0, 2, 1, 3) for x in (k, v))
    o, lse = _attend(qs, ks, vs, visible, st["scale"])
    at = torch.arange(q.shape[0], device=dev)
    seq = torch.searchsorted(cu_q, at, right=True) - 1
    pos = at - cu_q[seq]
    o = o.view(B, Hkv, G, Lq, D)[seq, :, :, pos].reshape(-1, Hq, D)
    return o.to(torch.bfloat16), lse.view(B, Hkv, G, Lq)[seq, :, :, pos].reshape(-1, Hq)


def _slots(st):
    """The page and the place in it of every token that is written or read back."""
    cu, kv_len, page = st["cu"].long(), st["kv_len"].long(), st["page"]
    at = torch.arange(st["k"].shape[0], device=cu.device)
    seq = torch.searchsorted(cu, at, right=True) - 1
    pos = kv_len[seq] - (cu[seq + 1] - at)
    return st["table"].long()[seq, pos // page], pos % page


def _plain_cache(st):
    where, place = _slots(st)
    got = []
    for pages, scales, x in ((st["k_pages"], st["k_scale"], st["k"]), (st["v_pages"], st["v_scale"], st["v"])):
        if scales is None:
            pages[where, :, place] = x
            got.append(pages[where, :, place])
        else:
            c, s = _quantise(x)
            pages.view(torch.uint8)[where, :, place] = c.view(torch.uint8)
            scales[where, :, place] = s
            got.append(_values(pages.view(torch.uint8)[where, :, place].view(torch.float8_e4m3fn), scales[where, :, place]).to(torch.bfloat16))
    return tuple(got)


def _plain_decode(st):
    q, kv_len, page, table = st["q"], st["kv_len"].long(), st["page"], st["table"].long()
    B, Hq, Hkv, D, n = q.shape[0], st["Hq"], st["Hkv"], st["D"], st["max_total"]
    if st["k"] is not None:
        live = st["live"]                                                              # (a slot without a sequence appends nothing)
        last = kv_len[live] - 1
        where, place = table[live, last // page], last % page
        st["k_pages"][where, :, place], st["v_pages"][where, :, place] = st["k"][live], st["v"][live]
    ks, vs = (
        (p[table].float() if s is None else _values(p.view(torch.uint8)[table].view(torch.float8_e4m3fn), s[table]))
        .permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)[:, :, :n] for p, s in ((st["k_pages"], st["k_scale"]), (st["v_pages"], st["v_scale"])))
    visible = (torch.arange(n, device=q.device) < kv_len[:, None])[:, None, None]
    o, lse = _attend(q.float().view(B, Hkv, Hq // Hkv, D), ks, vs, visible, st["scale"])
    return o.reshape(B, Hq, D).to(torch.bfloat16), lse.reshape(B, Hq)


# ---------------------------------------------------------------------------------------------------------------- one pass

def run(state):
    st, kind = state, state["kind"]
    if own:
        eng = st["eng"]
        if kind == "prompt":
            return eng.prompt(st["q"], st["k"], st["v"], st["cu_q"], st["cu_k"], out=st["out"], lse=st["lse"])
        if kind == "cache":
            eng.paged_write(st["cache"], st["k"], st["v"], st["cu"], st["table"], st["kv_len"])
            return eng.paged_read(st["cache"], st["cu"], st["table"], st["kv_len"], st["k_out"], st["v_out"])
        got = eng.paged_decode(st["q"], st["k"], st["v"], st["cache"], st["table"], st["kv_len"], out=st["out"], lse=st["lse"])
    else:
        if kind == "prompt":
            return _plain_prompt(st)
        if kind == "cache":
            return _plain_cache(st)
        got = _plain_decode(st)
    return (*got, st["k_pages"], st["v_pages"]) if st["k"] is not None else tuple(got)   # a step that appends has changed the cache


def work(case):
    new, ctx = _lens(case)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    total = [a + b for a, b in zip(new, ctx)]
    row = Hkv * (D + 1 if case["e4m3"] else 2 * D)             # a token's keys, or its values, in the cache
    if case["kind"] == "prompt":
        seen = sum(a * b + a * (a + 1) // 2 for a, b in zip(new, ctx))
        return {"bytes": sum(new) * Hq * (4 * D + 4) + sum(total) * Hkv * 4 * D, "flops": 4 * D * Hq * seen}
    if case["kind"] == "cache":
        return {"bytes": sum(new) * (4 * row + 8 * Hkv * D), "flops": 0}
    added = sum(n > 0 for n in new) * Hkv * 4 * D if case["append"] else 0
    return {"bytes": 2 * sum(total) * row + len(new) * Hq * (4 * D + 4) + 2 * added, "flops": 4 * D * Hq * sum(total)}


# ---------------------------------------------------------------------------------------------------------------- 64 bits

def _softmax_rows(q, k, v, scale, first_last):
    """Attention of the rows q [r, d] over k, v [n, d] in 64 bits; row i sees the keys 0 .. first_last[i]."""
    logits = (q @ k.T) * scale
    hidden = torch.arange(k.shape[0], device=k.device)[None, :] > first_last[:, None]
    logits[hidden] = -math.inf
    lse = torch.logsumexp(logits, dim=1)
    w = torch.exp(logits - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
    return w @ v, lse


def _e4m3_of(x):
    """The values that 8-bit pages hold for rows x, in 64 bits: rounded to four significant bits, ties to even."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    power = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 448))
    power = torch.where(top > 448 * torch.exp2(power), power + 1, power)
    power = torch.where(top <= 448 * torch.exp2(power - 1), power - 1, power).clamp(-127, 120)
    y = x / torch.exp2(power)
    size = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -20)))
    size = torch.where(torch.exp2(size) > y.abs(), size - 1, size).clamp(min=-6)
    step = torch.exp2(size - 3)
    return torch.round(y / step) * step * torch.exp2(power)


def exact(case, seed):
    new, ctx = _lens(case)
    total = [a + b for a, b in zip(new, ctx)]
    Hq, Hkv, D, page = case["Hq"], case["Hkv"], case["D"], case["page"]
    G, scale, st = Hq // Hkv, D ** -0.5, prepare(case, seed)
    if case["kind"] == "cache":
        if not case["e4m3"]:
            return st["k"].double(), st["v"].double()
        return _e4m3_of(st["k"]), _e4m3_of(st["v"])
    rows = sum(new) if case["kind"] == "prompt" else len(new)
    out = torch.zeros(rows, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((rows, Hq), -math.inf, dtype=torch.float64, device="cuda")
    at_q = at_k = 0
    for i, (a, n) in enumerate(zip(new, total)):
        if case["kind"] == "prompt":
            mine = slice(at_q, at_q + a)
            q, k, v = st["q"][mine].double(), st["k"][at_k:at_k + n].double(), st["v"][at_k:at_k + n].double()
            last = torch.arange(a, device="cuda") + (n - a)
            at_q, at_k = at_q + a, at_k + n
        else:
            mine = slice(i, i + 1)
            if n == 0:
                continue
            pages = st["table"][i, :-(-n // page)].long()
            q = st["q"][mine].double()
            k, v = (st[x + "_pages"].view(torch.uint8)[pages].view(st[x + "_pages"].dtype).to(torch.float64) for x in "kv")
            if case["e4m3"]:
                k, v = (y * torch.exp2(st[x + "_scale"][pages].double() - 127)[..., None] for x, y in (("k", k), ("v", v)))
            k, v = (y.permute(0, 2, 1, 3).reshape(-1, Hkv, D)[:n].clone() for y in (k, v))
            if case["append"]:
                k[n - 1], v[n - 1] = st["k"][i].double(), st["v"][i].double()
                st["k_pages"][pages[-1], :, (n - 1) % page], st["v_pages"][pages[-1], :, (n - 1) % page] = st["k"][i], st["v"][i]
            last = torch.tensor([n - 1], device="cuda")
        for h in range(Hq):
            out[mine, h], lse[mine, h] = _softmax_rows(q[:, h], k[:, h // G], v[:, h // G], scale, last)
    if case["kind"] == "decode" and case["append"]:
        return out, lse, st["k_pages"].double(), st["v_pages"].double()
    return out, lse
