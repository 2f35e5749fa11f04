"""Host-side check of how many steps keys take and how tiles are laid along a line and cut, compiled out of the kernel's source: every step of every
tile lies in one run, whatever the lengths."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_08077_b200", "csrc")

PROGRAM = r"""
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#define __device__
#define __host__
#define __forceinline__ inline
using std::max; using std::min;
struct FastDiv { int d; int div(int n) const { return n / d; } };
template <bool kPaged> struct PromptSeq { int q0, k0, nq, nk, off, nt, b; };
struct PromptGeom { int T, Hkv, most_steps, window, sinks; FastDiv div_w; };
%s
struct Line {
%s
    long long place, cost;
%s
};
%s
int main() {
    if (prompt_steps(0) != 0 || prompt_steps(1) != 1 || prompt_steps(128) != 1 || prompt_steps(129) != 2 || prompt_steps(2147483632) != 16777216) return 1;
    srand(7);
    for (int round = 0; round < 4000; ++round) {
        PromptGeom g;
        g.T = 8 + rand() %% 121;
        g.Hkv = 1 + rand() %% 4;
        g.div_w.d = 2 * g.T;
        g.most_steps = rand() %% 2 ? kPromptMostSteps : 2 + rand() %% 40;
        PromptSeq<true> q;
        q.nq = 1 + rand() %% 3000;
        q.nk = rand() %% 8 == 0 ? 0 : rand() %% 2 ? rand() %% 4000 : rand() %% 200000;
        q.off = q.nk - q.nq;
        q.nt = (q.nq + 2 * g.T - 1) / (2 * g.T);
        long long sum = 0;
        for (int t = 0; t <= q.nt; ++t) {                     // closed form against the sum
            if (Line::length(g, q, t) != sum) { printf("length %%d of %%d %%d %%d %%d\n", t, q.nq, q.nk, g.T, g.most_steps); return 2; }
            if (t < q.nt) sum += Line::cost_of(g, q, t);
        }
        const int pairs = 1 + rand() %% 74;
        const PromptRuns runs(sum, pairs);
        if (runs.begin(0) != 0 || runs.begin(pairs) != sum) return 3;
        long long place = 0;
        for (int t = 0; t < q.nt; ++t) {                      // the parts of a tile, run by run, are its steps
            Line l;
            l.place = place;
            l.cost = Line::cost_of(g, q, t);
            const int n = 1 + rand() %% 300;
            int at = 0;
            for (int r = 0; r < pairs; ++r) {
                const int a = l.steps_before(runs.begin(r), n), b = l.steps_before(runs.begin(r + 1), n);
                if (b < a) return 4;
                if (b > a) {
                    if (a != at) return 5;
                    at = b;
                }
            }
            if (at != n) return 6;
            place += l.cost;
        }
    }
    return 0;
}
"""


def test_line_and_runs(tmp_path):
    text = open(os.path.join(CSRC, "attn_prompt.cuh")).read()

    def part(begin, end):
        a = text.index(begin)
        return text[a:text.index(end, a)]
    constants = part("constexpr int kPromptMostSteps", "// The order of the items") + part("constexpr int kPromptAhead", "struct PromptLine")
    statics = part("    static __device__ __forceinline__ long long limit(", "    __device__ __forceinline__ bool load(const PromptGeom& g, int c, int lane)")
    before = part("    __device__ __forceinline__ int steps_before(", "};\n// The line's runs")
    runs = part("struct PromptRuns {", "\ntemplate <int D, int kKeys>")
    prog = tmp_path / "line.cpp"
    prog.write_text(PROGRAM % (constants, statics, before, runs))
    exe = str(tmp_path / "line")
    subprocess.run(["g++", "-std=c++17", "-O1", str(prog), "-o", exe], check=True)
    got = subprocess.run([exe], capture_output=True, text=True)
    assert got.returncode == 0, (got.returncode, got.stdout)
    assert re.search(r"kPromptMostSteps = 1 << 24", text)
