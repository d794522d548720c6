"""What can be held to without a GPU, from the kernels' sources: paths that a run takes only when a bounded wait gives up, and orders
that a run keeps or breaks by the compiler's choice."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_36301_b200", "csrc")


def source(name):
    """A file without its comments."""
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", ["more_experts_sm100.cu", "more_combine.cu"])
def test_warps_that_stay_together_give_up_together(name):
    """All lanes of a warp wait in these kernels, and go on to instructions that need all of them."""
    text = source(name)
    assert len(re.findall(r"\bmbar_wait_warp\(", text)) >= 2
    assert not re.findall(r"\bmbar_wait\(", text)
    common = source("sm100_common.cuh")
    assert re.search(r"bool mbar_wait_warp\([^)]*\)\s*\{\s*return __all_sync\(0xffffffffu, mbar_wait\(", common)


def test_a_ring_settles_before_its_cta_ends():
    """A CTA that gave up a wait has copies under way into its shared memory: it goes on to its end only behind a pause for them."""
    text = source("more_combine.cu")
    kernels = [k for k in re.split(r"__global__", text)[1:] if "mbar_wait_warp(" in k]
    assert len(kernels) == 2
    for k in kernels:
        loop = k.index("mbar_wait_warp(")
        assert "settle(abort_flag);" in k[loop:] and not re.search(r"\breturn\b", k[loop:k.index("settle(abort_flag);")])
    assert re.search(r"void settle\([^)]*\)\s*\{\s*__syncthreads\(\);\s*if \(!\*abort_flag\) return;.*__nanosleep.*__syncthreads\(\);", text, re.S)


def test_kernels_that_begin_early_promise_nothing_about_their_inputs():
    """A kernel that may begin before the one in front of it has ended does not take what that one writes as __restrict__ (or read-only),
    which would let its loads move in front of the wait."""
    seen = 0
    for name in sorted(os.listdir(CSRC)):
        text = source(name)
        for kernel in re.split(r"__global__", text)[1:]:
            signature, body = kernel.split("{", 1)
            if "wait_for_previous();" in body:
                seen += 1
                assert "__restrict__" not in signature and "__ldg(" not in body and "ld.global.nc" not in body, (name, signature)
    assert seen >= 4
