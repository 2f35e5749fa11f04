"""More of what a program does with text beside the video, as a set of measurable cases: what happens to queries and keys between
the projection and the attention, and attention over a paged cache by more than one new token, or by a window of it.

  rotate  queries and keys of every head divided by the root of their mean square (where the model does so) and rotated by
          their positions; the pairs of a head follow one axis of positions each (time, height, width of a patch)
  append  the same on the way into the cache: rotated queries come back, rotated keys and the values go into their pages, as
          bf16 or as 8-bit floats with a power of two per token and head
  chunk   causal attention of several new tokens per sequence over the pages of its cache (their own keys and values are there
          already), all of it or a window of the last tokens and the first few
  decode  attention of one new token per sequence over its window and the first few

With a window of w tokens and s first ones, the token at position p sees the positions j <= p with j > p - w or j < s.

8-bit pages: a row x of head_dim values is held as e4m3 codes c and one byte s, x ~ c * 2^(s - 127), with the smallest
power of two for which the row's largest magnitude is at most 448 (s in 0 .. 247).
"""
from __future__ import annotations

import math

import torch

own = False

_EPS = 1e-6
_BASE = {
    "kind": "chunk", "lens": "41", "ctx": "", "Hq": 28, "Hkv": 4, "D": 128, "page": 16, "e4m3": False,
    "window": 0, "sinks": 0,                                                     # chunk, decode
    "sections": "64", "theta": 1e6, "adjacent": False, "norm": False,            # rotate, append: pairs of each axis
}


def _case(name, **kw):
    return {**_BASE, **kw, "name": name}


def listed():
    return [
        # A video of the benchmark's layer and the text behind it: patches have a time, a row and a column.  Heads with norms.
        _case("rotate_video_16k", kind="rotate", lens="16512", sections="16,24,24", norm=True),
        # An odd number of tokens of the smaller heads, of which a part is rotated, neighbouring values as pairs.
        _case("rotate_part_d64", kind="rotate", lens="701", Hq=16, Hkv=4, D=64, sections="16", theta=1e4, adjacent=True),
        # One decode step of sixteen conversations about long videos: latency.
        _case("append_step", kind="append", lens="1x16", ctx="131000x16", sections="16,24,24", page=64),
        # Ordinary prompts of odd lengths into 8-bit pages, small heads with norms.
        _case("append_prompts_e4m3_d64", kind="append", lens="700,1,2049,333,64,1535", ctx="0,15,100,0,64,0", Hq=16, Hkv=4, D=64, e4m3=True,
              sections="32", theta=1e4, norm=True),
        # The tokens of a long video of the benchmark into the cache.
        _case("append_video_64k", kind="append", lens="65536", sections="16,24,24", page=64, norm=True),
        # One short turn of a single conversation: latency.
        _case("chunk_turn", lens="41", ctx="503"),
        # What a scheduler packs into one step: first and later chunks of prompts beside single new tokens.
        _case("chunk_batch_mixed", lens="512,1,37,1024,1,1,300,1", ctx="0,5000,8192,1024,131,77,4000,16000"),
        # Proposed tokens of sixteen long conversations, looked at together, in 8 bits.
        _case("chunk_proposed_b16_e4m3", lens="5,4,5,5,1,5,5,3,5,5,5,2,5,5,5,5", page=64, e4m3=True,
              ctx="32768,20000,40000,31111,8192,50000,32768,1025,16384,28000,65536,700,30000,45000,12345,32000"),
        # A chunk of questions and documents behind a long video, in 8 bits.
        _case("chunk_long_e4m3", lens="2048", ctx="65536", page=64, e4m3=True),
        # Chunks of long prompts of the smaller heads, whose tokens look back a part of the way.
        _case("chunk_window_d64", lens="4096,1000,1,777", ctx="4096,20000,12000,0", Hq=16, Hkv=4, D=64, page=32, window=1024, sinks=4),
        # Serving: conversations of any length, one slot of the batch unused, with a window.
        _case("decode_window_ragged", kind="decode", window=1024, sinks=4,
              lens="5000,1,17,8192,300,0,4097,2500,64,1023,777,6000,128,129,3333,50,2048,1500,900,7000,15,16,450,5555"),
        # Serving: sixteen conversations of the longest length in 8 bits, with a wide window.
        _case("decode_window_128k_b16_e4m3", kind="decode", lens="131584x16", page=64, e4m3=True, window=16384, sinks=64),
    ]


_HEADS = [(4, 4, 64), (16, 4, 64), (8, 2, 128), (16, 2, 128), (28, 4, 128), (28, 4, 128)]
_MAX_ROTATE = 65536 * 36 * 128
_MAX_PAIRS = 28 * 2048 * 66560           # (query head, row, key) triples of the largest chunk case
_MAX_CACHE = 16 * 131584 * 4 * 128       # tokens * kv heads * head_dim of the largest decode case


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["rotate", "append", "append", "chunk", "chunk", "chunk", "decode"])
        Hq, Hkv, D = rng.choice(_HEADS)
        c = {**_BASE, "kind": kind, "Hq": Hq, "Hkv": Hkv, "D": D, "page": rng.choice([16, 16, 32, 64, 128]),
             "e4m3": kind != "rotate" and rng.random() < 0.5}
        n = _log_uniform(rng, 1, 24)
        top = _log_uniform(rng, 2, {"rotate": 65536, "append": 65536, "chunk": 8192, "decode": 131072}[kind])
        lens = [max(1, _log_uniform(rng, max(1, top // 16), top)) for _ in range(n)]
        ctx = [0] * n
        if kind in ("append", "chunk"):
            far = _log_uniform(rng, 1, 65536)
            ctx = [rng.choice([0, _log_uniform(rng, max(1, far // 16), far)]) for _ in range(n)]
        if kind in ("rotate", "append"):
            c["norm"] = rng.random() < 0.5
            c["adjacent"] = rng.random() < 0.3
            c["theta"] = rng.choice([1e4, 5e5, 1e6])
            half = D // 2
            c["sections"] = rng.choice([str(half), str(half), str(half // 2), f"{half // 4},{half // 8 * 3},{half // 8 * 3}", f"{half // 2},{half // 2}"])
            if sum(lens) * (Hq + 2 * Hkv) * D > _MAX_ROTATE or sum(a + b for a, b in zip(lens, ctx)) * Hkv * D > _MAX_CACHE // 4:
                continue
        else:
            if kind == "decode" or rng.random() < 0.5:
                c["window"], c["sinks"] = _log_uniform(rng, 16, 16384), rng.choice([0, 0, 1, 4, 64, 200])
            if kind == "decode" and n > 1 and rng.random() < 0.3:
                lens[rng.randrange(n)] = 0
            if kind == "chunk" and sum(Hq * a * (a + b) for a, b in zip(lens, ctx)) > _MAX_PAIRS:
                continue
            if n * (max(lens) + max(ctx)) * Hkv * D > _MAX_CACHE // (4 if kind == "chunk" else 1):
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


def _frequencies(case):
    """Radians per position and the axis of every pair."""
    sections = _numbers(case["sections"])
    n = sum(sections)
    return [case["theta"] ** (-i / n) for i in range(n)], [a for a, m in enumerate(sections) for _ in range(m)]


def _positions(new, ctx, axes, device):
    """int32 [axes, tokens].  One axis: places in the sequence.  Several: a single new token stands where the text behind a video does, the
    same on all axes; more are patches, frame by frame in 16 rows of 16, from a sequence's first place on."""
    got = []
    for n, before in zip(new, ctx):
        i = torch.arange(n, device=device)
        if axes == 1 or n == 1:
            got.append((i + before).expand(axes, n))
        else:
            got.append(torch.stack([i // 256, i // 16 % 16, i % 16][:axes]) + before)
    return torch.cat(got, 1).to(torch.int32).contiguous()


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    kind, Hq, Hkv, D, page = case["kind"], case["Hq"], case["Hkv"], case["D"], case["page"]
    new, ctx = _lens(case)
    total = [a + b for a, b in zip(new, ctx)]
    n = sum(new)
    randn = lambda *s: torch.randn(*s, generator=g, device=dev).to(torch.bfloat16)  # noqa: E731
    st = {"kind": kind, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "scale": D ** -0.5, "new": new, "total": total,
          "window": case["window"], "sinks": case["sinks"], "adjacent": case["adjacent"]}
    if kind in ("rotate", "append"):
        qkv = randn(n, Hq + 2 * Hkv, D)                       # what one projection gives
        grow = torch.exp2(torch.randint(-3, 4, (n, 1, 1), generator=g, device=dev).float()).to(torch.bfloat16)
        qkv.mul_(grow)
        st["q"], st["k"], st["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        freq, axis = _frequencies(case)
        st["freq"], st["axis"] = torch.tensor(freq, dtype=torch.float64, device=dev), torch.tensor(axis, device=dev)
        st["positions"] = _positions(new, ctx, max(axis) + 1, dev)
        near_one = lambda: (1 + 0.2 * torch.randn(D, generator=g, device=dev)).to(torch.bfloat16)  # noqa: E731
        st["q_norm"], st["k_norm"] = (near_one(), near_one()) if case["norm"] else (None, None)
        st["q_out"] = torch.empty(n, Hq, D, dtype=torch.bfloat16, device=dev)
        st["k_out"] = torch.empty(n, Hkv, D, dtype=torch.bfloat16, device=dev)
        st["v_out"] = torch.empty_like(st["k_out"])
    if kind != "rotate":
        # a pool of pages in no order, the sequences' pages scattered over it
        per = [-(-m // page) for m in total]
        n_pages, width = sum(per) + 3, max(per)
        order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
        table = torch.zeros(len(per), width, dtype=torch.int32, device=dev)
        at = 0
        for i, m in enumerate(per):
            table[i, :m] = order[at:at + m]
            at += m
        st["table"], st["kv_len"], st["cu"] = table, torch.tensor(total, dtype=torch.int32, device=dev), _cumulative(new, dev)
        k, v = randn(n_pages, Hkv, page, D), randn(n_pages, Hkv, page, D)
        if case["e4m3"]:
            (st["k_pages"], st["k_scale"]), (st["v_pages"], st["v_scale"]) = _quantise(k), _quantise(v)
        else:
            st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"] = k, v, None, None
    if kind in ("chunk", "decode"):
        rows = n if kind == "chunk" else len(new)
        st["q"] = randn(rows, Hq, D)
        st["out"] = torch.empty(rows, Hq, D, dtype=torch.bfloat16, device=dev)
        st["lse"] = torch.empty(rows, Hq, dtype=torch.float32, device=dev)
    if own:
        from paper_2604_08077_b200 import binding
        st["eng"] = binding.AdaSAttn(cube=(4, 4, 4), n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, top_p=0.9)
        if kind in ("rotate", "append"):
            st["rotary"] = binding.Rotary(D, sections=_numbers(case["sections"]), theta=case["theta"], adjacent=case["adjacent"])
        if kind != "rotate":
            st["cache"] = binding.PagedCache(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
    return st


# ---------------------------------------------------------------------------------------------------------------- plain forms

def _turned(x, weight, cos, sin, adjacent):
    """Rows x [n, h, D] with their norm and rotation, in the type of cos; the first 2 * pairs values of a head are rotated."""
    x = x.to(cos.dtype)
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * weight.to(cos.dtype)
    pairs = cos.shape[1]
    c, s = cos[:, None], sin[:, None]
    if adjacent:
        a, b = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = x[..., :pairs], x[..., pairs:2 * pairs]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([turned, x[..., 2 * pairs:]], -1)


def _angles(st):
    """[tokens, pairs] in 64 bits: far positions times small frequencies."""
    return st["positions"].double()[st["axis"]].T * st["freq"]


def _plain_rotated(st):
    a = _angles(st)
    cos, sin = torch.cos(a).float(), torch.sin(a).float()
    return _turned(st["q"], st["q_norm"], cos, sin, st["adjacent"]), _turned(st["k"], st["k_norm"], cos, sin, st["adjacent"])


def _slots(st):
    """The page and the place in it of every new token."""
    cu, kv_len, page = st["cu"].long(), st["kv_len"].long(), st["page"]
    at = torch.arange(int(st["q"].shape[0]), device=cu.device)
    seq = torch.searchsorted(cu, at, right=True) - 1
    pos = kv_len[seq] - (cu[seq + 1] - at)
    return st["table"].long()[seq, pos // page], pos % page


def _plain_append(st):
    q, k = _plain_rotated(st)
    where, place = _slots(st)
    got = [q.to(torch.bfloat16)]
    for pages, scales, x in ((st["k_pages"], st["k_scale"], k), (st["v_pages"], st["v_scale"], st["v"])):
        if scales is None:
            pages[where, :, place] = x.to(torch.bfloat16)
            got.append(pages)
        else:
            c, s = _quantise(x)
            pages.view(torch.uint8)[where, :, place] = c.view(torch.uint8)
            scales[where, :, place] = s
            got.append(_values(pages.view(torch.uint8)[where, :, place].view(torch.float8_e4m3fn), scales[where, :, place]).to(torch.bfloat16))
    return tuple(got)


def _hidden(first, rows, keys, window, sinks):
    """Which of the positions `keys` the tokens at first .. first + rows - 1 do not see."""
    p = first + torch.arange(rows, device=keys.device)[:, None]
    hidden = keys > p
    if window:
        hidden |= (keys <= p - window) & (keys >= sinks)
    return hidden


def _seen(first, n, window, sinks, device):
    """The positions below n that some token from `first` on sees."""
    lo = max(0, first + 1 - window) if window else 0
    return torch.cat([torch.arange(min(sinks, lo), device=device), torch.arange(lo, n, device=device)])


def _cached(st, b, keys, dtype):
    """Keys and values [Hkv, keys, D] of sequence b."""
    where, place = st["table"][b].long()[keys // st["page"]], keys % st["page"]
    got = []
    for pages, scales in ((st["k_pages"], st["k_scale"]), (st["v_pages"], st["v_scale"])):
        if scales is None:
            x = pages[where, :, place].to(dtype)
        else:
            x = pages.view(torch.uint8)[where, :, place].view(torch.float8_e4m3fn).to(dtype)
            x = x * torch.exp2(scales[where, :, place].to(dtype) - 127)[..., None]
        got.append(x.transpose(0, 1))
    return got


def _attention(st, dtype):
    """Outputs and logarithms of the sums of all rows in `dtype`, sequence by sequence and kv head by kv head."""
    q, Hkv, D = st["q"], st["Hkv"], st["D"]
    G = st["Hq"] // Hkv
    out = torch.zeros(q.shape, dtype=dtype, device=q.device)
    lse = torch.full(q.shape[:2], -math.inf, dtype=dtype, device=q.device)
    at = 0
    for b, (n_new, n) in enumerate(zip(st["new"], st["total"])):
        r = n_new if st["kind"] == "chunk" else 1
        rows = slice(at, at + r)
        at += r
        if n == 0:
            continue
        keys = _seen(n - r, n, st["window"], st["sinks"], q.device)
        hidden = _hidden(n - r, r, keys, st["window"], st["sinks"]).repeat(G, 1)
        k, v = _cached(st, b, keys, dtype)
        for h in range(Hkv):
            qh = q[rows, h * G:(h + 1) * G].to(dtype).transpose(0, 1).reshape(G * r, D)
            s = torch.matmul(qh * st["scale"], k[h].T).masked_fill_(hidden, -math.inf)
            m = s.amax(-1, keepdim=True)
            s.sub_(m).exp_()
            l = s.sum(-1, keepdim=True)
            out[rows, h * G:(h + 1) * G] = (torch.matmul(s, v[h]) / l).view(G, r, D).transpose(0, 1)
            lse[rows, h * G:(h + 1) * G] = (m + torch.log(l)).view(G, r).T
    return out, lse


# ---------------------------------------------------------------------------------------------------------------- one pass

def run(state):
    st, kind = state, state["kind"]
    if own:
        eng = st["eng"]
        if kind == "rotate":
            return eng.rotate(st["q"], st["k"], st["positions"], st["rotary"], q_norm=st["q_norm"], k_norm=st["k_norm"], eps=_EPS,
                              q_out=st["q_out"], k_out=st["k_out"])
        if kind == "append":
            q = eng.paged_append(st["cache"], st["q"], st["k"], st["v"], st["cu"], st["table"], st["kv_len"], st["rotary"], positions=st["positions"],
                                 q_norm=st["q_norm"], k_norm=st["k_norm"], eps=_EPS, q_out=st["q_out"])
            if st["k_scale"] is None:
                return q, st["k_pages"], st["v_pages"]
            return (q, *eng.paged_read(st["cache"], st["cu"], st["table"], st["kv_len"], st["k_out"], st["v_out"]))   # what the codes stand for
        if kind == "chunk":
            return eng.paged_prompt(st["q"], st["cache"], st["cu"], st["table"], st["kv_len"], window=st["window"], sinks=st["sinks"], out=st["out"], lse=st["lse"])
        return eng.paged_decode(st["q"], None, None, st["cache"], st["table"], st["kv_len"], window=st["window"], sinks=st["sinks"], out=st["out"], lse=st["lse"])
    if kind == "rotate":
        return tuple(x.to(torch.bfloat16) for x in _plain_rotated(st))
    if kind == "append":
        return _plain_append(st)
    out, lse = _attention(st, torch.float32)
    return out.to(torch.bfloat16), lse


def work(case):
    new, ctx = _lens(case)
    kind, Hq, Hkv, D = case["kind"], case["Hq"], case["Hkv"], case["D"]
    n = sum(new)
    row = Hkv * (D + 1 if case["e4m3"] else 2 * D)            # a token's keys, or its values, in the cache
    turned = n * (Hq + Hkv) * (3 * 2 * sum(_numbers(case["sections"])) + (4 * D if case["norm"] else 0))
    places = 4 * n * len(_numbers(case["sections"]))
    if kind == "rotate":
        return {"bytes": n * (Hq + Hkv) * 4 * D + places, "flops": turned}
    if kind == "append":
        back = 2 * n * (row + 2 * Hkv * D) if case["e4m3"] else 0
        return {"bytes": n * (Hq * 4 * D + 2 * (2 * Hkv * D + row)) + places + back, "flops": turned}
    w, s = case["window"], case["sinks"]
    if kind == "decode":
        ctx, new = [max(m - 1, 0) for m in new], [min(m, 1) for m in new]
    keys = pairs = 0
    for a, b in zip(new, ctx):
        if a == 0:
            continue
        m = a + b
        lo = max(0, b + 1 - w) if w else 0
        keys += min(s, lo) + m - lo
        p = torch.arange(b, m, dtype=torch.int64)
        out_of_window = (p + 1 - w).clamp(min=0) if w else torch.zeros_like(p)
        pairs += int((p + 1 - out_of_window + out_of_window.clamp(max=s)).sum())
    rows = n if kind == "chunk" else len(new)
    return {"bytes": 2 * keys * row + rows * Hq * (4 * D + 4), "flops": 4 * D * Hq * pairs}


# ---------------------------------------------------------------------------------------------------------------- 64 bits

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


def _rotation_matrix_rows(x, weight, positions, freq, axis, adjacent):
    """Rows x [n, h, D] in 64 bits: every pair is a complex number, multiplied by e^(i angle)."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + _EPS) * weight.double()
    pairs = freq.numel()
    angle = positions.double()[axis].T * freq
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    if adjacent:
        z = torch.view_as_complex(x[..., :2 * pairs].reshape(*x.shape[:2], pairs, 2).contiguous()) * turn
        first = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(x[..., :pairs].contiguous(), x[..., pairs:2 * pairs].contiguous()) * turn
        first = torch.cat([z.real, z.imag], -1)
    return torch.cat([first, x[..., 2 * pairs:]], -1)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("rotate", "append"):
        q = _rotation_matrix_rows(st["q"], st["q_norm"], st["positions"], st["freq"], st["axis"], st["adjacent"])
        k = _rotation_matrix_rows(st["k"], st["k_norm"], st["positions"], st["freq"], st["axis"], st["adjacent"])
        if kind == "rotate":
            return q, k
        if case["e4m3"]:
            return q, _e4m3_of(k), _e4m3_of(st["v"])
        got = [q]
        cu, at = st["cu"].tolist(), []
        for b, (n_new, n) in enumerate(zip(st["new"], st["total"])):
            pos = torch.arange(n - n_new, n, device="cuda")
            at.append(st["table"][b].long()[pos // st["page"]] * st["page"] + pos % st["page"])
        at = torch.cat(at)
        for pages, x in ((st["k_pages"], k), (st["v_pages"], st["v"].double())):
            flat = pages.double().permute(0, 2, 1, 3).reshape(-1, st["Hkv"], st["D"])
            flat[at] = x[:cu[-1]]
            got.append(flat.view(pages.shape[0], st["page"], st["Hkv"], st["D"]).permute(0, 2, 1, 3))
        return tuple(got)
    # attention row by row of the definition: softmax over what a row sees, head by head
    q, Hq, Hkv, D = st["q"].double(), st["Hq"], st["Hkv"], st["D"]
    out = torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    at = 0
    for b, (n_new, n) in enumerate(zip(st["new"], st["total"])):
        r = n_new if kind == "chunk" else 1
        rows, at = slice(at, at + r), at + r
        if n == 0:
            continue
        pages = st["table"][b, :-(-n // st["page"])].long()
        k, v = (st[x + "_pages"].view(torch.uint8)[pages].view(st[x + "_pages"].dtype).to(torch.float64) for x in "kv")
        if case["e4m3"]:
            k, v = (y * torch.exp2(st[x + "_scale"][pages].double() - 127)[..., None] for x, y in (("k", k), ("v", v)))
        k, v = (y.permute(0, 2, 1, 3).reshape(-1, Hkv, D)[:n] for y in (k, v))
        p, j = torch.arange(n - r, n, device=q.device)[:, None], torch.arange(n, device=q.device)
        sees = j <= p
        if case["window"]:
            sees &= (j > p - case["window"]) | (j < case["sinks"])
        for h in range(Hq):
            logits = (q[rows, h] @ k[:, h * Hkv // Hq].T * st["scale"]).masked_fill_(~sees, -math.inf)
            lse[rows, h] = torch.logsumexp(logits, 1)
            out[rows, h] = torch.softmax(logits, 1) @ v[:, h * Hkv // Hq]
    return out, lse
