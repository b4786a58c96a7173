"""Rules that the kernels of the tree operators keep (source checks, on the CPU; the
failures they exclude would be a hang or a stale value).

A wait that can give up is decided by the warp as a whole, as in the prompt kernels
(tests/test_wait_uniformity.py); and as dependent launches they start while the kernel that
writes their inputs may still run, so nothing is read through the non-coherent path
(tests/test_dependent_launch_loads.py) and every kernel waits before its first access.
"""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2309_08168_gb300", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_waits_are_decided_by_the_warp():
    src = source("tree_attn.cu")
    calls = [m.start() for m in re.finditer(r"\bmb_wait\(", src) if not src[:m.start()].endswith("bool ")]
    assert len(calls) == 1 and src[:calls[0]].endswith("__all_sync(0xffffffffu, ")
    assert len(re.findall(r"\bmb_try\(", src)) == 2 and len(re.findall(r"\bwait\(", src)) >= 12


@pytest.mark.parametrize("name", ["tree_attn.cu", "tree_attn.cuh", "tree_few.cu", "tree_ops.cu", "tree_ops.cuh", "tree_sched.cuh"])
def test_no_non_coherent_loads(name):
    src = source(name)
    assert "global.nc" not in src and "__ldg(" not in src and "__restrict__" not in src


@pytest.mark.parametrize("name,kernels", [("tree_attn.cu", ["attn_kernel", "join_kernel"]), ("tree_few.cu", ["few_kernel"]), ("tree_ops.cu", ["plan_kernel", "rope_kernel", "commit_kernel"])])
def test_kernels_wait_for_the_one_before(name, kernels):
    src = source(name)
    for k in kernels:
        body = src[re.search(r"\b%s\(" % k, src).start():]
        body = body[:body.index("\n}\n")]
        before = body[:body.index("pdl_wait()")]
        assert "pdl_launch_dependents()" in body and "__ldcg" not in before and "return" not in before, k
