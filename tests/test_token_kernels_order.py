"""What the token kernels (csrc/dc_sample.cu, dc_token_attn.cuh) do in which order, read from their sources: faults of this kind are races and waits that a run
rarely shows."""
import os
import re

import pytest

import paper_2609_35115_b200 as dc

CSRC = os.path.join(os.path.dirname(dc.__file__), "csrc")


def kernel(file, name):
    """The body of a kernel, without comments."""
    with open(os.path.join(CSRC, file)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    at = re.search(r"__global__[^;{]*\b%s\(" % name, text).end()
    at = text.index("{", at)
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i + 1]
    raise AssertionError(name)


def test_no_cta_of_a_sampling_cluster_leaves_while_another_may_read_its_memory():
    """Every way out of the kernel ends at a cluster barrier that is passed, not only arrived at."""
    body = kernel("dc_sample.cu", "sample_kernel")
    passed = r"(?:if \(a\.splits > 1\) )?(?:cluster_or_block_sync\(a\.splits\)|ptx::cluster_wait\(\));\s*"
    ways = [m.start() for m in re.finditer(r"\n\s*return;", body)] + [len(body) - 1]
    assert len(ways) == 4
    for end in ways:
        assert re.search(passed + r"$", body[:end].rstrip() + "\n"), body[max(0, end - 300):end]


@pytest.mark.parametrize("file,name", [("dc_token_attn.cuh", "attend_chunk_kernel"), ("dc_flow.cu", "flow_gemm_kernel"), ("dc_flow.cu", "flow_attn_kernel")])
def test_dependents_start_behind_the_allocation_of_tensor_memory(file, name):
    """A dependent grid may allocate before it waits for this one: it must not find columns that a CTA of this one has yet to take."""
    body = re.sub(r"if \(p\.empty\) \{[^}]*\}", "", kernel(file, name))      # (the form that does nothing)
    allocated = max(m.start() for m in re.finditer(r"tmem_alloc(_pair)?\(", body))
    assert body.count("pdl_launch") == 1 and allocated < body.index("__syncthreads();", allocated) < body.index("pdl_launch")


def test_tensor_memory_is_given_back_before_a_cta_waits_for_its_cluster():
    """A CTA of the cluster may be waiting for columns that another kernel's CTA pair holds, and the pair for this CTA's."""
    body = kernel("dc_token_attn.cuh", "attend_chunk_kernel")
    assert body.rindex("tmem_dealloc") < body.index("cluster_arrive") < body.index("cluster_wait")
    assert body.rindex("tmem_ld64(lane_base + CH_O") < body.index("cluster_arrive")


@pytest.mark.parametrize("file,name", [("dc_token_attn.cuh", "attend_chunk_kernel"), ("dc_token_cache.cu", "attend_step_kernel"), ("dc_sample.cu", "sample_kernel")])
def test_whole_warps_meet_at_the_cluster_barriers(file, name):
    """Behind branches that a warp's lanes may have taken apart they come together before they arrive."""
    with open(os.path.join(CSRC, file)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    arrivals = [m.start() for m in re.finditer(r"ptx::cluster_arrive\(\);", text)]
    assert arrivals and "cluster_arrive" in (kernel(file, name) if name != "sample_kernel" else text)
    for at in arrivals:
        assert re.search(r"__syncwarp\(\);\s*$", text[:at]), text[max(0, at - 200):at]
