"""The operators of ssd_ops.h on the CPU: what the library exports, the layout of
their structures, the calls that they refuse before a device is touched, and
the frequencies of ssd_rope_init.
"""
import ctypes
import math
import os
import re

import numpy as np
import pytest

import tree_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ssd():
    import __graft_entry__ as g
    g._lib_builder().build()
    import paper_2309_08168_gb300 as m
    return m


def test_exports_every_declared_operator(ssd):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ssd_ops.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\bint (ssd_\w+)\s*\(", src)))
    assert sorted(ssd.OPERATOR_EXPORTS) == names and len(names) == 6
    for n in names:
        assert hasattr(ctypes.CDLL(ssd.LIB_PATH), n), n


def test_structures_match_the_header(ssd, tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#include "ssd.h"\n#include "ssd_ops.h"\n#include <stdio.h>\n#include <stddef.h>\n'
                   'int main(void) { printf("%zu %zu %zu %zu %zu %zu", sizeof(ssd_pages), offsetof(ssd_pages, layer_stride), sizeof(ssd_batch),'
                   ' offsetof(ssd_batch, row_start), sizeof(ssd_rope), offsetof(ssd_rope, turns)); return 0; }\n')
    import subprocess
    exe = tmp_path / "s"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert got == [ctypes.sizeof(ssd.ssd_pages), ssd.ssd_pages.layer_stride.offset, ctypes.sizeof(ssd.ssd_batch),
                   ssd.ssd_batch.row_start.offset, ctypes.sizeof(ssd.ssd_rope), ssd.ssd_rope.turns.offset]


P = 0x10000  # an aligned address; never read on the host


def pages(ssd, **kw):
    f = dict(k=P, v=P, dtype=ssd.SSD_F16, n_layers=2, n_pages=10, n_kv_heads=2, page_size=16, head_dim=64,
             layer_stride=10 * 2 * 16 * 64, page_stride=2 * 16 * 64, head_stride=16 * 64, pos_stride=64)
    f.update(kw)
    return ssd.ssd_pages(*f.values())


def batch(ssd, **kw):
    f = dict(n_requests=2, n_rows=6, max_rows=3, max_blocks=4, row_start=P, lens=P, block_table=P)
    f.update(kw)
    return ssd.ssd_batch(*f.values())


BAD_PAGES = [dict(k=None), dict(v=P + 8), dict(dtype=0), dict(head_dim=96), dict(n_layers=0), dict(n_kv_heads=0), dict(page_size=24), dict(page_size=0),
             dict(page_size=131072), dict(n_pages=0), dict(n_pages=1 << 27), dict(pos_stride=60), dict(pos_stride=32), dict(page_stride=-64),
             dict(head_stride=8), dict(layer_stride=0), dict(page_stride=1 << 38)]
BAD_BATCH = [dict(row_start=None), dict(lens=None), dict(block_table=None), dict(n_requests=0), dict(n_requests=4097), dict(n_rows=-1), dict(max_rows=0),
             dict(max_blocks=0)]


def attention(ssd, pg=None, bt=None, **kw):
    f = dict(layer=1, dtype=ssd.SSD_F32, n_heads=4, q=P, qs=256, masks=P, words=1, scale=0.125, out=2 * P, os=256, ws=P, wb=1 << 30, status=None, stream=None)
    f.update(kw)
    return ssd.lib.ssd_tree_attention(bt or batch(ssd), pg or pages(ssd), *f.values())


def rope(ssd, pg=None, rp=None, **kw):
    f = dict(dtype=ssd.SSD_F32, n_rows=3, n_heads=4, q=P, qs=256, k=P, ks=128, v=P, vs=128, pos=P, slots=P, out=P, os=256, stream=None)
    f.update(kw)
    layer = f.pop("layer", 0)
    return ssd.lib.ssd_rope_kv(pg or pages(ssd), layer, rp or ssd.ssd_rope_init(64), *f.values())


def plan(ssd, bt=None, **kw):
    f = dict(page=16, n_pages=10, parents=P, held=P, held_out=2 * P, ring=P, ends=P, ends_out=2 * P, slots=P, positions=P, masks=P, words=1, status=None, stream=None)
    f.update(kw)
    return ssd.lib.ssd_tree_plan(bt or batch(ssd), *f.values())


def commit(ssd, pg=None, bt=None, **kw):
    f = dict(parents=P, tokens=P, target=P, acc=P, nxt=P, lens_out=2 * P, path=P, emitted=P, stream=None)
    f.update(kw)
    return ssd.lib.ssd_tree_commit(bt or batch(ssd), pg or pages(ssd), *f.values())


def refused(ssd, rc, call, code=None):
    assert rc == (code or ssd.SSD_ERR_INVALID_ARG), (rc, ssd.ssd_last_error())
    assert ssd.ssd_last_error().startswith(call + ": ")


@pytest.mark.parametrize("bad", BAD_PAGES, ids=str)
def test_bad_caches_are_refused(ssd, bad):
    refused(ssd, attention(ssd, pages(ssd, **bad)), "ssd_tree_attention")
    refused(ssd, rope(ssd, pages(ssd, **bad)), "ssd_rope_kv")
    refused(ssd, commit(ssd, pages(ssd, **bad)), "ssd_tree_commit")


@pytest.mark.parametrize("bad", BAD_BATCH, ids=str)
def test_bad_batches_are_refused(ssd, bad):
    refused(ssd, attention(ssd, bt=batch(ssd, **bad)), "ssd_tree_attention")
    refused(ssd, plan(ssd, batch(ssd, **bad)), "ssd_tree_plan")
    refused(ssd, commit(ssd, bt=batch(ssd, **bad)), "ssd_tree_commit")


def test_null_structures_are_refused(ssd):
    assert ssd.lib.ssd_tree_plan(None, 16, 10, *[P] * 9, 1, None, None) == ssd.SSD_ERR_INVALID_ARG
    assert ssd.lib.ssd_tree_commit(None, None, *[P] * 8, None) == ssd.SSD_ERR_INVALID_ARG
    assert ssd.lib.ssd_tree_attention_workspace(64, None) == ssd.SSD_ERR_INVALID_ARG
    assert ssd.lib.ssd_rope_init(64, 0, 0, 1e4, 1, 0, 0, 0, 1, None) == ssd.SSD_ERR_INVALID_ARG
    import ctypes as c
    assert ssd.lib.ssd_tree_attention_workspace(96, c.byref(c.c_size_t())) == ssd.SSD_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(layer=2), dict(layer=-1), dict(dtype=2), dict(dtype=7), dict(n_heads=3), dict(n_heads=0), dict(q=None), dict(out=None),
                                 dict(ws=None), dict(ws=P + 4), dict(qs=255), dict(qs=128), dict(os=258), dict(q=P + 8), dict(out=P), dict(scale=0.0),
                                 dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(words=0), dict(words=5), dict(masks=None)], ids=str)
def test_attention_refuses(ssd, bad):
    refused(ssd, attention(ssd, **bad), "ssd_tree_attention")


def test_attention_says_when_the_workspace_is_short(ssd):
    refused(ssd, attention(ssd, wb=0), "ssd_tree_attention", ssd.SSD_ERR_CAPACITY)


@pytest.mark.parametrize("bad", [dict(layer=2), dict(dtype=2), dict(n_rows=-1), dict(n_heads=0), dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(slots=None),
                                 dict(out=None), dict(qs=250), dict(ks=64), dict(vs=130), dict(k=P + 4), dict(os=512)], ids=str)
def test_rope_refuses(ssd, bad):
    refused(ssd, rope(ssd, **bad), "ssd_rope_kv")


def test_rope_wider_than_the_head_is_refused(ssd):
    refused(ssd, rope(ssd, rp=ssd.ssd_rope_init(128)), "ssd_rope_kv")


@pytest.mark.parametrize("bad", [dict(page=8), dict(n_pages=0), dict(held=None), dict(held_out=None), dict(held_out=P), dict(ring=None), dict(ends=None), dict(ends_out=None),
                                 dict(ends_out=P), dict(slots=None), dict(positions=None), dict(masks=None), dict(words=0), dict(words=5), dict(parents=None)], ids=str)
def test_plan_refuses(ssd, bad):
    refused(ssd, plan(ssd, **bad), "ssd_tree_plan")


@pytest.mark.parametrize("bad", [dict(tokens=None), dict(target=None), dict(acc=None), dict(nxt=None), dict(lens_out=None), dict(lens_out=P), dict(path=None), dict(emitted=None)],
                         ids=str)
def test_commit_refuses(ssd, bad):
    refused(ssd, commit(ssd, **bad), "ssd_tree_commit")


def test_empty_calls_need_no_device(ssd):
    assert rope(ssd, n_rows=0, q=None) == ssd.SSD_OK
    assert attention(ssd, bt=batch(ssd, n_rows=0), q=None) == ssd.SSD_OK


@pytest.mark.parametrize("bad", [dict(rot_dim=24), dict(rot_dim=0), dict(rot_dim=144), dict(theta=1.0), dict(theta=math.inf), dict(theta=math.nan), dict(scaling=3), dict(scaling=-1),
                                 dict(scaling=1, factor=0.5), dict(factor=math.nan), dict(amplitude=0.0), dict(amplitude=1e39), dict(scaling=2, factor=2.0),
                                 dict(scaling=2, factor=2.0, original_len=100, slow=4.0, fast=4.0), dict(scaling=2, original_len=100, slow=-1.0)], ids=str)
def test_rope_init_refuses(ssd, bad):
    with pytest.raises(ssd.SSDError) as e:
        ssd.ssd_rope_init(**{"rot_dim": 64, **bad})
    assert e.value.code == ssd.SSD_ERR_INVALID_ARG and "ssd_rope_init" in str(e.value)


@pytest.mark.parametrize("rot,theta,kw", [(128, 1e4, {}), (16, 5e5, {}), (48, 1e4, dict(scaling=1, factor=4.0)),
                                          (128, 1e4, dict(scaling=2, factor=8.0, original_len=4096, slow=1.0, fast=32.0)),
                                          (64, 1e6, dict(scaling=2, factor=1.5, original_len=8192, slow=0.0, fast=2.0))])
def test_rope_frequencies(ssd, rot, theta, kw):
    r = ssd.ssd_rope_init(rot, theta, **kw)
    f = ref.frequencies(rot, theta, kw.get("scaling", 0), kw.get("factor", 1.0), kw.get("original_len", 0.0), kw.get("slow", 1.0), kw.get("fast", 32.0))
    got = np.array([r.turns[i] / 2.0**64 for i in range(64)])
    # both sides round a handful of times in 64 bits; turns are multiples of 2^-64, off by half of that
    np.testing.assert_allclose(got[:rot // 2], f / (2 * math.pi), rtol=1e-14, atol=2.0**-65)
    assert not got[rot // 2:].any() and r.rot_dim == rot and r.amplitude == 1.0


def test_reference_plan_is_consistent():
    """The oracle on a batch worked by hand: a chain, an ended request, one that does not fit, a tree."""
    table = np.full((4, 4), -9, np.int32)
    table[0, 0], table[1, :2], table[2, :2], table[3, 0] = 4, [2, 6], [0, 1], 3
    ring = np.array([9, 7, 8, 5, -9, -9, -9, -9, -9, -9], np.int32)
    got = ref.plan([0, 3, 3, 20, 23], np.array([15, -1, 32, 16]), np.array([-1, 0, 0] + [-1] * 17 + [-1, 0, 1]), table, np.array([1, 2, 2, 1]), ring,
                   np.array([1, 3]), 16, 10, 23, 1)
    assert got["slots"][:3].tolist() == [4 * 16 + 15, 7 * 16, 7 * 16 + 1]
    assert got["positions"][:3].tolist() == [15, 16, 16]
    assert got["masks"][:3, 0].tolist() == [1, 3, 5]
    assert (got["slots"][3:20] == -1).all() and got["status"] == 1  # two pages more: none is left after request 0's and 3 has to wait
    assert got["ends"].tolist() == [2, 5] and got["ring"][3:5].tolist() == [2, 6]
    assert got["held"].tolist() == [2, 0, 2, 1] and got["slots"][20] == -1


def test_stalls_without_a_limit_are_refused(ssd):
    for bad in (0.0, -1.0, 11.0, math.nan):
        with pytest.raises(ssd.SSDError):
            ssd.ssd_debug_tree_stall(0, bad)
    ssd.ssd_debug_tree_stall(-1)


def test_commit_refuses_results_in_the_place_of_inputs(ssd):
    """Every result in every input's place, and in each other's; with arrays of their own the call gets as far as the device."""
    own = {n: (i + 10) * P for i, n in enumerate(("parents", "tokens", "target", "acc", "nxt", "lens_out", "path", "emitted"))}
    b = batch(ssd, row_start=P, lens=2 * P, block_table=3 * P)
    assert commit(ssd, bt=b, **own) != ssd.SSD_OK and "arrays of their own" not in ssd.ssd_last_error()
    results = ("acc", "nxt", "lens_out", "path", "emitted")
    for r in results:
        for at in (P, 2 * P, 3 * P, *(own[x] for x in own if x != r)):
            refused(ssd, commit(ssd, bt=b, **{**own, r: at}), "ssd_tree_commit")
            assert "arrays of their own" in ssd.ssd_last_error()
    assert "arrays of their own" not in (commit(ssd, bt=b, **{**own, "parents": None}), ssd.ssd_last_error())[1]
