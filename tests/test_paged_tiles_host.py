"""Host-side check of how many tiles a sequence has, and how many boxes or quarters of a tile hold a token (paged_decode.cuh, paged_tiles
and paged_pieces), up to the longest one that a block table has room for.

The two routines are read out of the source, compiled for the host with overflow of signed integers trapped, and compared with 64-bit
arithmetic; nothing else in the source rounds a number of tokens up to tiles."""
import os
import re
import subprocess

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_08077_b200", "csrc", "paged_decode.cuh")

PROGRAM = r"""
#include <cstdint>
#include <cstdio>
#define __host__
#define __device__
%s
%s
int main() {
    long long seen = 0;
    for (int tile = 64; tile <= 128; tile *= 2)
        for (long long around = 0; around <= (1ll << 31); around = around ? around * 2 : 1)
            for (long long x = around - 300; x <= around + 300; ++x) {
                if (x < 0 || x > INT32_MAX) continue;
                const int n = (int)x;
                if (paged_tiles(n, tile) != (x + tile - 1) / tile) return 1;
                for (int size = 16; size <= tile && n > 0; size *= 2) {
                    const long long want = (x + size - 1) / size < tile / size ? (x + size - 1) / size : tile / size;
                    if (paged_pieces(n, tile, size) != want) return 2;
                }
                ++seen;
            }
    std::printf("%%lld\n", seen);
    return 0;
}
"""


def test_tiles_of_the_longest_sequences(tmp_path):
    text = open(SRC).read()
    parts = [re.search(r"__host__ __device__ constexpr int %s\(.*?\}\n" % name, text).group(0) for name in ("paged_tiles", "paged_pieces")]
    assert not re.search(r"kTile - 1\) / kTile|sub - 1\) / sub|kWarpKeys - 1\) / kWarpKeys", text)
    prog = tmp_path / "tiles.cpp"
    prog.write_text(PROGRAM % tuple(parts))
    exe = str(tmp_path / "tiles")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error", str(prog), "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True)
    assert res.returncode == 0 and int(res.stdout) > 10000, res.returncode
