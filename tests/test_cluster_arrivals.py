"""Arrivals at a barrier of the other CTA of a pair say what they order: TMEM
(relaxed: tcgen05 fences on both sides do it), or what threads of this CTA have
stored (a release for the cluster, met by waits that acquire for it).  The plain
remote arrival, whose release ends at the CTA, is for stages that the copies' and
MMAs' own completion orders."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_23805_gb300", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_chunk_kernel_orders_what_it_stores():
    text = source("kv_chunk.cu")
    assert "mbar_arrive_remote" not in text
    # relaxed: weights and outputs, after a fence of the tensor core's accesses
    for m in re.finditer(r"mbar_arrive_relaxed\((\w+)", text):
        assert m.group(1) in ("lead_pfull", "lead_ofree")
        assert "tc_fence_before();" in text[max(0, m.start() - 120):m.start()]
    # everything else crosses by a release after a wait in the same CTA
    crossing = re.findall(r"mbar_arrive_cluster\(", text)
    assert len(crossing) == 1
    at = text.index("mbar_arrive_cluster(")
    assert "mbar_wait_warp(bar, parity & 1" in text[at - 200:at]
    # and the MMA warps acquire for the cluster
    assert re.search(r"auto wait = \[&\]\(uint64_t\* bar, uint32_t parity\) \{ return mbar_wait_warp<true>\(", text)


def test_scopes_in_the_helpers():
    text = source("internal.cuh")
    assert "mbarrier.arrive.release.cluster.shared::cluster.b64" in text
    assert "mbarrier.arrive.relaxed.cluster.shared::cluster.b64" in text
    assert "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64" in text
