"""The operators of ssd_step.h on the CPU: how large a workspace is asked for."""
import ctypes

import pytest

import test_step_ops as ops


@pytest.fixture(scope="module")
def ssd():
    import __graft_entry__ as g
    g._lib_builder().build()
    import paper_2309_08168_gb300 as m
    return m


@pytest.mark.parametrize("d,f,e", [(4096, 14336, 8), (5120, 13824, 16), (64, 48, 8), (2048, 768, 128), (4104, 1416, 64), (512, 65536, 3), (8, 16384, 1024), (65536, 4096, 2), (320, 8192, 200)])
@pytest.mark.parametrize("dtype", ["SSD_F16", "SSD_BF16"])
def test_a_workspace_for_many_rows_is_enough_for_few(ssd, d, f, e, dtype):
    m = ops.moe(ssd, d=d, f=f, n_experts=e, gs=d * f, us=d * f, ds=d * f, dtype=getattr(ssd, dtype))

    def size(n, k):
        b = ctypes.c_size_t()
        assert ssd.lib.ssd_moe_workspace(m, n, k, b) == ssd.SSD_OK
        return b.value
    rows = [*range(0, 140), *range(200, 1025, 59), 1024]
    got = [[size(n, k) for k in range(1, 17)] for n in rows]
    for i, x in enumerate(got):
        assert x == sorted(x), rows[i]
        if i:
            assert all(a <= b for a, b in zip(got[i - 1], x)), rows[i]
    # what each pair's activations and at least one sum of its results take
    for n, x in zip(rows, got):
        assert all(b >= n * k * (4 * f + 4 * d) for k, b in zip(range(1, 17), x))
