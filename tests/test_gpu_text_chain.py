"""The operators together, as a program uses them: a conversation in chunks and single tokens against one pass over all of it; a video whose queries and
keys are rotated by time, height and width on the way into its prefill."""
import numpy as np
import pytest
import torch

import oracle
from paper_2604_08077_b200 import binding, inputs
from text_util import BF16_HALF, assert_close, assert_lse, engine, scattered, sequence_values
from window_util import attend_masked, hidden_from, rotated

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 5)])
def test_a_conversation(window, sinks, e4m3):
    """Two conversations side by side: a prompt, a longer turn, three single tokens; the outputs of every step are those of 64 bits over what the pages hold."""
    g = torch.Generator().manual_seed(3)
    Hq, Hkv, D, page = 14, 2, 128, 32
    eng = engine(Hq, Hkv, D)
    steps = [(100, 7), (37, 300), (1, 1), (1, 1), (1, 1)]
    total = [sum(s[b] for s in steps) for b in range(2)]
    table, n_pages = scattered(g, [-(-n // page) for n in total])
    cache = eng.paged_cache(n_pages, page, e4m3=e4m3)
    rope, w = binding.Rotary(D, theta=1e6), (1 + 0.1 * torch.randn(D, generator=g)).to(torch.bfloat16).cuda()
    lens = [0, 0]
    for new in steps:
        lens = [a + b for a, b in zip(lens, new)]
        x = torch.randn(sum(new), Hq + 2 * Hkv, D, generator=g).to(torch.bfloat16).cuda()
        q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        cu, kv_len = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
        q_rot = eng.paged_append(cache, q, k, v, cu, table, kv_len, rope, q_norm=w, k_norm=w)
        if new == (1, 1):
            out, lse = eng.paged_decode(q_rot, None, None, cache, table, kv_len, window=window, sinks=sinks, want_lse=True)
        else:
            out, lse = eng.paged_prompt(q_rot, cache, cu, table, kv_len, window=window, sinks=sinks, want_lse=True)
        assert eng.text_status() == 0
        for b, rows in ((0, slice(0, new[0])), (1, slice(new[0], sum(new)))):
            pos = torch.arange(lens[b] - new[b], lens[b], device="cuda")
            turned, tol = rotated(q[rows], w, pos, [1e6 ** (-i / 64) for i in range(64)], [0] * 64, False, 1e-6)
            assert_close(q_rot[rows], turned, tol + BF16_HALF * turned.abs() + 1e-30, "q")
            keys, values = sequence_values(cache, table, b, lens[b])
            want, wl, otol, ltol = attend_masked(q_rot[rows], keys, values, hidden_from(lens[b] - new[b], new[b], lens[b], window, sinks), D ** -0.5)
            if e4m3:                                             # q in two parts: 2^-18 of its largest magnitude, as a score
                e = q_rot[rows].double().abs().amax(-1) * 2.0 ** -18 * keys.abs().sum(-1).amax() * D ** -0.5
                otol, ltol = otol + (2 * e * values.abs().amax())[..., None], ltol + e
            assert_close(out[rows], want, otol, "out")
            assert_lse(lse[rows], wl, ltol)


def test_a_video_rotated_by_its_axes():
    """rotate() in place on a fused projection, then the prefill: the oracle on the rotated rows, and these against 64 bits."""
    wl = inputs.config1()
    B, S, Hq, D = wl.q.shape
    Hkv = wl.k.shape[2]
    frames, gh, gw = wl.T, wl.H, wl.W
    i = torch.arange(S, device="cuda")
    patch = i < frames * gh * gw
    behind = max(frames, gh, gw) + i - frames * gh * gw           # text: the same on all axes
    pos = torch.stack([torch.where(patch, x, behind) for x in (i // (gh * gw), i // gw % gh, i % gw)]).to(torch.int32).contiguous()
    eng = binding.AdaSAttn(cube=wl.cube, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, top_p=wl.top_p)
    sections = [8, 12, 12]
    rope = binding.Rotary(D, sections=sections, theta=1e4)
    q, k, v = wl.q.cuda(), wl.k.cuda(), wl.v.cuda()
    for b in range(B):
        before = q[b].clone(), k[b].clone()
        eng.rotate(q[b], k[b], pos, rope, q_out=q[b], k_out=k[b])
        for got, x in ((q[b], before[0]), (k[b], before[1])):
            want, tol = rotated(x, None, pos, [1e4 ** (-j / 32) for j in range(32)], [a for a, m in enumerate(sections) for _ in range(m)], False, 0.0)
            assert_close(got, want, tol + BF16_HALF * want.abs() + 1e-30, "rotated")
    eng.partition(wl.B, wl.T, wl.H, wl.W, wl.n_text)
    out, bitmap, _ = eng.forward(q, k, v, wl.n_text, want_selection=True)
    sh = oracle.shape_of(wl, top_p=float(np.float32(wl.top_p)))
    res = oracle.rows(sh, q.cpu(), k.cpu(), wl.v, oracle.all_rows(sh))
    words = bitmap.cpu().numpy().view(np.uint32)
    sel = ((words[..., None] >> np.arange(32, dtype=np.uint32)) & 1).reshape(*words.shape[:-1], -1)[..., :sh.N].reshape(-1, sh.N)
    sure = res["margin"] >= 1e-6
    assert (sel == res["sel"])[sure].all()
    got = out.float().cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, D)
    assert np.abs(got - res["out"])[(sel == res["sel"]).all(axis=1)].max() < 2e-2
