"""A serving step in a graph (tokens on the way into their pages, attention of several and of one by a window over long caches that are cut and joined),
replayed with other tokens and lengths, against 64 bits; two objects at work at once."""
import pytest
import torch

from paper_2604_08077_b200 import binding
from test_gpu_paged_prompt import ints, pool, rand
from text_util import assert_close, assert_lse, engine, sequence_values
from window_util import attend_masked, hidden_from

pytestmark = pytest.mark.gpu
WINDOW, SINKS = 6000, 140


def check_rows(got, lse, q, keys, values, first, window, sinks, e4m3):
    r, D = q.shape[0], q.shape[-1]
    want, wl, tol, ltol = attend_masked(q, keys, values, hidden_from(first, r, first + r, window, sinks), D ** -0.5)
    if e4m3:                                                     # q in two parts: 2^-18 of its largest magnitude, as a score
        e = q.double().abs().amax(-1) * 2.0 ** -18 * keys.abs().sum(-1).amax() * D ** -0.5
        tol, ltol = tol + (2 * e * values.abs().amax())[..., None], ltol + e
    assert_close(got, want, tol, "out")
    assert_lse(lse, wl, ltol)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D", [(28, 4, 128), (8, 2, 64)])
def test_append_chunk_and_decode_in_one_graph(Hq, Hkv, D, e4m3):
    g = torch.Generator().manual_seed(312)
    page, room = 32, [12000, 9000, 2500]
    eng = engine(Hq, Hkv, D)
    table, cache = pool(g, room, page, Hkv, D, e4m3)
    rotary = binding.Rotary(D)
    # sequences 0 and 1 get several tokens, sequence 2 one by the decode
    q, k, v = rand(g, 46, Hq, D), rand(g, 46, Hkv, D), rand(g, 46, Hkv, D)
    cu, lens = ints([0, 41, 45, 46]), ints([5000, 300, 700])

    def step():
        qo = eng.paged_append(cache, q, k, v, cu, table, lens, rotary)
        several = eng.paged_prompt(qo[:45], cache, cu[:3], table[:2], lens[:2], window=WINDOW, sinks=SINKS, want_lse=True)
        one = eng.paged_decode(qo[45:], None, None, cache, table[2:], lens[2:], window=1000, sinks=SINKS, want_lse=True)
        return qo, *several, *one
    step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            qo, out, lse, out1, lse1 = step()
    torch.cuda.synchronize()
    for kv in ([12000, 9000, 2500], [41, 8999, 1], [7013, 130, 1003]):
        lens.copy_(ints(kv))
        for x in (q, k, v):
            x.copy_(rand(g, *x.shape))
        for x in (out, lse, out1, lse1):
            x.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert eng.text_status() == 0
        for b, rows in ((0, slice(0, 41)), (1, slice(41, 45))):
            keys, values = sequence_values(cache, table, b, kv[b])
            check_rows(out[rows], lse[rows], qo[rows], keys, values, kv[b] - (rows.stop - rows.start), WINDOW, SINKS, e4m3)
        keys, values = sequence_values(cache, table, 2, kv[2])
        check_rows(out1, lse1, qo[45:], keys, values, kv[2] - 1, 1000, SINKS, False)


@pytest.mark.parametrize("e4m3", [False, True])
def test_two_objects_at_once(e4m3):
    """Objects with workspaces of their own, on streams of their own, over one cache that both only read: what each gives alone."""
    g = torch.Generator().manual_seed(313)
    Hq, Hkv, D, page, kv = 28, 4, 128, 64, [30000, 9000]
    table, cache = pool(g, kv, page, Hkv, D, e4m3)
    lens = ints(kv)
    work = []
    for seed, new in ((1, [5, 4]), (2, [60, 9])):
        eng, q = engine(Hq, Hkv, D), rand(g, sum(new), Hq, D)
        cu = ints([0, new[0], sum(new)])

        def calls(eng=eng, q=q, cu=cu):
            a, la = eng.paged_prompt(q, cache, cu, table, lens, want_lse=True)
            b, lb = eng.paged_decode(q[:2], None, None, cache, table, lens, window=20000, sinks=64, want_lse=True)
            c, lc = eng.paged_prompt(q, cache, cu, table, lens, window=4000, sinks=200, want_lse=True)
            return a, la, b, lb, c, lc
        work.append((eng, calls, calls()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(12):
        for i, (_, calls, _) in enumerate(work):
            with torch.cuda.stream(streams[i]):
                got[i].append(calls())
    torch.cuda.synchronize()
    for i, (eng, _, want) in enumerate(work):
        assert eng.text_status() == 0
        for outs in got[i]:
            for a, b in zip(outs, want):
                assert torch.equal(a, b)
