"""Host-side check of which steps of a tile over pages are walked as masked ones, compiled out of the kernel's source: the walk from a masked step to
the next meets every masked step and no other, for whole tiles and for parts of them.  (The loader of V asks step by step, the warp that answers
for those steps walks: a step that only one of them takes for a masked one is never answered.)"""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_08077_b200", "csrc")

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#define __device__
#define __host__
#define __forceinline__ inline
using std::max; using std::min;
template <bool kPaged> struct PromptSeq { int q0, k0, nq, nk, off, nt, b; };
struct Pages { int page_shift; };
struct PromptGeom { int T, window, sinks, most_steps; Pages pages; };
%s
%s
struct Tile {
    int n_steps, step0, sink_steps, base, low_first, low_masked, first_masked;
%s
};
long long seen = 0, before_low = 0;                           // tiles; those whose first masked step lies in front of the window's lower border
int walk(const PromptGeom& g, const PromptSeq<true>& q, int tile) {
    const PromptSpan x(g, q, tile);
    const int cuts[] = {0, x.n / 3, x.n / 2, x.n - x.n / 4, x.n};      // whole, and parts as a run's ends leave them
    for (int a : cuts)
        for (int b : cuts) {
            if (b <= a) continue;
            Tile t = {b - a, a, x.sink_steps, x.base, x.low_first - a, x.low_masked - a, max(x.first_masked - a, 0)};
            for (int j = 0; j <= t.n_steps; ++j) {
                int want = j;
                while (want < t.n_steps && !t.masked(want)) ++want;
                if (t.next_masked(j) != want) {
                    printf("from step %%d of %%d on: %%d, not %%d (T %%d, tile %%d of %%d + %%d tokens, window %%d, sinks %%d, part from %%d)\n", j, t.n_steps, t.next_masked(j), want, g.T, tile,
                           q.off, q.nq, g.window, g.sinks, a);
                    return 1;
                }
            }
            ++seen;
            before_low += t.first_masked < t.low_first && t.low_first < t.low_masked;
        }
    return 0;
}
int main(int argc, char**) {
    PromptGeom g;
    g.most_steps = kPromptMostSteps;
    auto sequence = [&](int off, int nq) {
        PromptSeq<true> q = {};
        q.nq = nq;
        q.off = off;
        q.nk = off + nq;
        q.nt = (nq + 2 * g.T - 1) / (2 * g.T);
        return q;
    };
    const int groups[] = {1, 2, 4, 7, 16}, offs[] = {0, 1, 77, 100, 127, 128, 300, 1111}, news[] = {1, 40, 129, 256, 300, 700};
    const int windows[] = {0, 1, 8, 16, 48, 100, 128, 200, 257, 600}, sinks[] = {0, 1, 4, 127, 128, 129, 200, 255, 256, 300, 700};
    for (int group : groups)
        for (int shift = 4; shift <= 8; ++shift)
            for (int off : offs)
                for (int nq : news)
                    for (int w : windows)
                        for (int s : sinks) {
                            g.T = 128 / group;
                            g.pages.page_shift = shift;
                            g.window = w;
                            g.sinks = w ? s : 0;
                            const PromptSeq<true> q = sequence(off, nq);
                            for (int tile = 0; tile < q.nt; ++tile)
                                if (walk(g, q, tile)) return 1;
                        }
    srand(5);
    for (int round = 0; round < 200000; ++round) {
        g.T = 1 + rand() %% 128;
        g.pages.page_shift = 4 + rand() %% 5;
        g.window = rand() %% 8 ? 1 + rand() %% (1 << (1 + rand() %% 11)) : 0;
        g.sinks = g.window && rand() %% 4 ? rand() %% (1 << (1 + rand() %% 11)) : 0;
        const PromptSeq<true> q = sequence(rand() %% 3 ? rand() %% 1500 : 0, 1 + rand() %% 1200);
        if (walk(g, q, rand() %% q.nt)) return 1;
    }
    if (before_low < 1000 || seen < 1000000) { printf("%%lld of %%lld\n", before_low, seen); return 2; }
    return 0;
}
"""


def test_masked_steps_are_walked_one_and_all(tmp_path):
    text = open(os.path.join(CSRC, "attn_prompt.cuh")).read()

    def part(begin, end):
        a = text.index(begin)
        return text[a:text.index(end, a)]
    prog = tmp_path / "masked.cpp"
    prog.write_text(PROGRAM % (part("constexpr int kPromptMostSteps", "// The order of the items"), part("struct PromptSpan {", "// Few tiles over pages"),
                               part("    __device__ __forceinline__ int key_of(", "};\n\n// A sequence as a planner sees it")))
    exe = str(tmp_path / "masked")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", str(prog), "-o", exe], check=True)
    got = subprocess.run([exe], capture_output=True, text=True)
    assert got.returncode == 0, (got.returncode, got.stdout, got.stderr[-500:])
