"""Host-side check of the steps that a tile over pages takes, compiled out of the kernel's source: what a row sees lies in one step, what a step
without a mask holds is seen by every row, and nothing leaves 32 bits, whatever the window, the first tokens and the lengths."""
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
long long draw(long long most) {                              // 0 .. most, of every size
    const int bits = rand() %% 32;
    return min<long long>(((long long)rand() << 16 ^ rand()) & ((1ll << bits) - 1), most);
}
int main() {
    srand(3);
    for (int round = 0; round < 400000; ++round) {
        PromptGeom g;
        g.pages.page_shift = 4 + rand() %% 5;
        g.T = 1 + rand() %% 128;
        g.window = rand() %% 10 == 0 ? 0 : rand() %% 10 == 0 ? 2147483647 : 1 + (int)draw(2147483646);
        g.sinks = !g.window || rand() %% 3 == 0 ? 0 : rand() %% 10 == 0 ? 2147483647 : (int)draw(2147483647);
        const long long room = g.window ? 0x7fffff00ll : (0x7fffffffll >> g.pages.page_shift) << g.pages.page_shift;
        PromptSeq<true> q;
        q.nk = (int)(rand() %% 10 == 0 ? room - rand() %% 300 : draw(room));
        q.nq = 1 + (int)draw(100000);
        q.off = q.nk - q.nq;
        q.nt = (q.nq + 2 * g.T - 1) / (2 * g.T);
        const int tile = rand() %% q.nt;
        const long long most = g.window ? (long long)g.sinks / 128 + ((long long)g.window + 2 * g.T) / 128 + 3 : kPromptMostSteps;
        const PromptSpan x(g, q, tile);
        if (x.n < 1 || x.n > min<long long>(most, kPromptMostSteps)) { printf("%%d steps of %%lld\n", x.n, most); return 1; }
        Tile t = {x.n, 0, x.sink_steps, x.base, x.low_first, x.low_masked, x.first_masked};
        const int box = min(1 << g.pages.page_shift, 128);
        const long long p0 = q.off + 2ll * tile * g.T, p1 = min(p0 + 2 * g.T, (long long)q.nk) - 1;
        auto sees = [&](long long p, long long j) { return j >= 0 && j <= p && (!g.window || j > p - g.window || j < g.sinks); };
        const long long rows[] = {p0, p1, p0 + rand() %% (p1 - p0 + 1)};
        for (long long p : rows) {
            const long long keys[] = {0, g.sinks - 1ll, p - g.window + 1, p, p > 0 ? draw(p) : 0, x.base, x.base - 1ll};
            for (long long j : keys) {
                if (!sees(p, j)) continue;
                // the step that holds it, by halves of the steps before and from sink_steps on
                int held = 0;
                if (j < 128ll * x.sink_steps) held += j / 128 < x.n;
                if (j >= x.base && (j - x.base) / 128 < x.n - x.sink_steps) ++held;
                if (held != 1) { printf("key %%lld of row %%lld in %%d steps (window %%d, sinks %%d, off %%d)\n", j, p, held, g.window, g.sinks, q.off); return 2; }
                if (!(j < x.hi && (j >= x.lo || j < g.sinks))) return 3;
            }
        }
        const int steps[] = {0, x.n - 1, x.sink_steps, x.sink_steps - 1, x.low_masked, x.low_masked - 1, x.first_masked - 1, x.first_masked, rand() %% x.n};
        for (int j : steps) {
            if (j < 0 || j >= x.n) continue;
            const long long key = t.key_of(j);
            if (key < 0 || key %% box || key > 0x7fffffffll - 127 || (j && key < t.key_of(j - 1) + 128ll)) { printf("step %%d at %%lld\n", j, key); return 4; }
            if (t.masked(j)) continue;
            for (long long p : rows)
                if (!sees(p, key) || !sees(p, key + 127)) { printf("row %%lld, step %%d at %%lld\n", p, j, key); return 5; }
        }
    }
    return 0;
}
"""


def test_steps_of_a_tile(tmp_path):
    text = open(os.path.join(CSRC, "attn_prompt.cuh")).read()

    def part(begin, end):
        a = text.index(begin)
        return text[a:text.index(end, a)]
    prog = tmp_path / "span.cpp"
    prog.write_text(PROGRAM % (part("constexpr int kPromptMostSteps", "// The order of the items"), part("struct PromptSpan {", "// Few tiles over pages"),
                               part("    __device__ __forceinline__ int key_of(", "    // the first masked step")))
    exe = str(tmp_path / "span")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", str(prog), "-o", exe], check=True)
    got = subprocess.run([exe], capture_output=True, text=True)
    assert got.returncode == 0, (got.returncode, got.stdout, got.stderr[-500:])
