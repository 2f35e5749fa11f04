"""Host-side check of how the text operators' kernels end when a wait has expired: they stay until what they had started (copies into
shared memory, products) has landed, for a limited time.  No wait is made to expire on a GPU: the order is read out of the sources, and the
routine is compiled for the host against a clock of its own."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_08077_b200", "csrc")

PROGRAM = r"""
#include <cstdint>
#include <cstdio>
#define __device__
#define __forceinline__ inline
static uint64_t now = 5000, reads = 0;
static uint64_t global_timer_ns() { ++reads; return now += 1000; }
%s
int main() {
    volatile int flag = 0;
    settle_after_abort(&flag);
    if (reads != 0) return 1;                             // an ordinary end costs nothing
    flag = 1;
    const uint64_t t0 = now;
    settle_after_abort(&flag);
    if (now - t0 < kSettleNs || now - t0 > kSettleNs + 10000) return 2;
    return 0;
}
"""


def test_settling_is_bounded(tmp_path):
    text = open(os.path.join(CSRC, "tc_common.cuh")).read()
    body = re.search(r"constexpr uint64_t kSettleNs.*?\n\}\n", text, re.S).group(0)
    prog = tmp_path / "settle.cpp"
    prog.write_text(PROGRAM % body)
    exe = str(tmp_path / "settle")
    subprocess.run(["g++", "-std=c++17", "-O1", str(prog), "-o", exe], check=True)
    assert subprocess.run([exe]).returncode == 0


def test_kernels_settle_before_they_give_their_memory_up():
    prompt = open(os.path.join(CSRC, "attn_prompt.cuh")).read()
    end = prompt[prompt.index("// ---------------------------------------------------------------- teardown"):]
    assert 0 < end.index("settle_after_abort(abort_flag)") < end.index("cluster_sync()") < end.index("tmem_dealloc_pair")
    decode = open(os.path.join(CSRC, "paged_decode.cuh")).read()
    kernel = decode[decode.index("paged_decode_kernel(PageGeom p"):decode.index("constexpr int kJoinThreads")]
    assert kernel.rstrip("\n/ ").count("settle_after_abort(abort_flag)") == 1
    after = kernel[kernel.index("settle_after_abort(abort_flag)"):]
    assert re.match(r"settle_after_abort\(abort_flag\);[^\n]*\n\}", after)        # the last thing that the consumers do
