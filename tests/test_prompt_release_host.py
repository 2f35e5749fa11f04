"""Host-side check, by reading the source, of what one CTA of a pair tells the other: an arrival on the other CTA's barrier that stands for shared memory
that threads have written or waited for is a release at the cluster's scope, and the thread that reads behind it acquires at that scope."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_08077_b200", "csrc")


def lines_of(name):
    return open(os.path.join(CSRC, name)).read().split("\n")


def test_arrivals_on_the_other_ctas_barriers():
    lines = lines_of("attn_prompt.cuh")
    plain = [i for i, x in enumerate(lines) if "tc::mbar_arrive_cluster(" in x]
    assert plain
    for i in plain:
        before = "\n".join(lines[max(i - 8, 0):i])
        # nothing but counted bytes of a TMA load; tensor memory, behind its own fence; behind a fence of the cluster's scope
        loads = "mbar_arrive_cluster(bar0 + st * 8)" in lines[i] and "mbar_arrive_expect_tx(" in before
        tensor_memory = re.search(r"mbar_arrive_cluster\((p_bar0 \+ buf \* 8|o_free_bar)\)", lines[i]) and "tc::tc_fence_before_sync();" in before
        fenced = "fence.acq_rel.cluster" in lines[i - 1]
        assert loads or tensor_memory or fenced, f"line {i + 1}: {lines[i].strip()}"


def test_waits_for_the_other_ctas_threads():
    text = "\n".join(lines_of("attn_prompt.cuh"))
    issuer = text[text.index("// ------------------------------------------------------------ MMA issuer"):text.index("// ------------------------------------------------------------ softmax warps")]
    waits = re.findall(r"(mbar_wait(?:<\w+>)?|there)\(&sm\.(v_full|q_peer)\[[^;]*?\)( \|\||\)| &&|;)", issuer)
    assert len(waits) == 2 and {w[1] for w in waits} == {"v_full", "q_peer"}
    assert "tc::mbar_wait<true>(&sm.v_full[vst], vph, abort_flag)" in issuer
    assert re.search(r"there\(&sm\.q_peer\[kn & 1\], \(kn >> 1\) & 1, both\)", issuer) and "const std::true_type both;" in issuer
    common = "\n".join(lines_of("tc_common.cuh"))
    assert "mbarrier.try_wait.parity.acquire.cluster" in common and "mbarrier.test_wait.parity.acquire.cluster" in common
    assert "mbarrier.arrive.release.cluster.shared::cluster" in common
