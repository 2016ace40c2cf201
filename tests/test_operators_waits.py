"""Waits on the device have limits: a warp that leaves its tile loop because a wait ran out must not leave another one behind at a
barrier without a limit."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_20055_b200", "csrc")


def _source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_warps_that_may_give_up_meet_at_no_hardware_barrier():
    """The contraction of the linear cross entropy leaves its loops when a wait runs out; whole-block barriers stand before the
    first of them and after the last alone."""
    text = _source("xent_gemm.cu")
    assert not re.search(r"\bbar(rier)?\.(cta\.)?(sync|red)\b|__syncthreads_|__barrier_sync", text)
    body = text[text.index("xent_gemm_kernel("):text.index("typedef CUresult")]
    first, last = body.index("if (warp == 0) {\n"), body.rindex("tcgen05_fence_before();\n    __syncthreads();")
    assert "__syncthreads" not in body[first:last] and "cluster_sync_all" not in body[first:last]
    # the meeting of two epilogue warps waits as the pipelines do
    meet = text[text.index("bool pair_meet("):]
    assert "pipe_wait(" in meet[:meet.index("\n}\n")]
    assert body.count("if (!pair_meet(") == body.count("pair_meet(") == 2


def test_the_product_of_4_bit_layers_never_leaves_its_loops_early():
    """Its product warps meet at a hardware barrier, so none of them may return or break out before the last meeting."""
    text = _source("int4.cu")
    kernel = text[text.index("int4_matvec_kernel("):text.index("cert_status_t launch_matvec3")]
    consumers = kernel[kernel.index("const uint32_t low = in_register"):]
    assert "consumers_meet();" in consumers
    assert not re.search(r"\b(return|break|goto)\b", consumers)
