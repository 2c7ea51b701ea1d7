"""The sampling kernel touches no other CTA's shared memory before every CTA of
its cluster has started (CPU, by reading the source).  A CTA whose part is short
or whose neighbour is late reaches the exchange of the maxima first; what it
stores into a CTA that does not run yet is undefined."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_15171_gb300", "csrc")
REMOTE = r"\b(dsmem_addr|dsmem_st_f32|dsmem_st_s32|dsmem_ld_s32|st_cluster_u32|st_cluster_u64|ld_cluster_u32|" \
         r"ld_cluster_u64|atom_cluster_add|push_sums<|send)\b"


def _kernel(name, file):
    """Body of a kernel, comments removed."""
    with open(os.path.join(CSRC, file), encoding="utf-8") as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    at = re.search(r"__global__[^;{]*\b" + name + r"\(", text).start()
    begin = text.index("{", at)
    depth = 0
    for i in range(begin, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[begin:i + 1]
    raise AssertionError("no end of the kernel")


def test_sampling_waits_for_its_cluster_before_the_first_remote_access():
    body = _kernel("sample_kernel", "sample.cu")
    remote = re.search(REMOTE, body).start()
    before = body[:remote]
    # one arrival and one wait, in this order, both outside any branch or loop, and
    # no way out of the kernel before them
    assert before.count("cluster_arrive_relaxed()") == 1 and before.count("cluster_wait()") == 1
    assert before.index("cluster_arrive_relaxed()") < before.index("cluster_wait()")
    assert "cluster_sync_all()" not in before
    for call in ("cluster_arrive_relaxed();", "cluster_wait();"):
        line = next(x for x in before.splitlines() if call in x)
        assert line.strip() == call and line.startswith("    c"), line
    assert not re.search(r"^    (if[^\n]*)?return\b", before, re.M)
