"""The operators of ssd_step.h on the CPU: what the library exports, the layout of their structures, the calls that they
refuse before a device is touched, the axes of ssd_rope_axes_init, and source rules of dependent launches.
"""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest

import step_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2309_08168_gb300", "csrc")
P = 0x10000  # an aligned address; never read on the host
FAR = 1 << 24  # apart from it


@pytest.fixture(scope="module")
def ssd():
    import __graft_entry__ as g
    g._lib_builder().build()
    import paper_2309_08168_gb300 as m
    return m


def test_exports_every_declared_operator(ssd):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ssd_step.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\bint (ssd_\w+)\s*\(", src)))
    assert sorted(ssd.STEP_EXPORTS) == names
    for n in names:
        assert hasattr(ctypes.CDLL(ssd.LIB_PATH), n), n


@pytest.mark.parametrize("name", ["ssd_rope_axes", "ssd_head_norm", "ssd_logit_rules", "ssd_moe"])
def test_structures_match_the_header(ssd, tmp_path, name):
    s = getattr(ssd, name)
    fields = [f[0] for f in s._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include "ssd_step.h"\n#include <stdio.h>\n#include <stddef.h>\nint main(void) { printf("%zu", sizeof(' + name + "));"
                   + "".join(f' printf(" %zu", offsetof({name}, {f}));' for f in fields) + " return 0; }\n")
    exe = tmp_path / "s"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert got == [ctypes.sizeof(s)] + [getattr(s, f).offset for f in fields]


def refused(ssd, rc, call, code=None):
    assert rc == (code or ssd.SSD_ERR_INVALID_ARG), (rc, ssd.ssd_last_error())
    assert ssd.ssd_last_error().startswith(call + ": ")


# -- heads -----------------------------------------------------------------------

def pages(ssd, **kw):
    f = dict(k=P, v=P, dtype=ssd.SSD_F16, n_layers=2, n_pages=10, n_kv_heads=2, page_size=16, head_dim=64,
             layer_stride=10 * 2 * 16 * 64, page_stride=2 * 16 * 64, head_stride=16 * 64, pos_stride=64)
    f.update(kw)
    return ssd.ssd_pages(*f.values())


def heads(ssd, pg=None, rp=None, axes=None, norm=None, **kw):
    f = dict(dtype=ssd.SSD_F32, n_rows=3, n_heads=4, q=P, qs=256, k=2 * P, ks=128, v=3 * P, vs=128, pos=P, slots=P, out=FAR, os=256, stream=None)
    f.update(kw)
    layer = f.pop("layer", 0)
    return ssd.lib.ssd_norm_rope_kv(pg or pages(ssd), layer, rp or ssd.ssd_rope_init(64), axes, norm, *f.values())


@pytest.mark.parametrize("bad", [dict(layer=2), dict(layer=-1), dict(dtype=2), dict(dtype=7), dict(n_rows=-1), dict(n_heads=0), dict(n_heads=65537), dict(q=None), dict(k=None),
                                 dict(v=None), dict(pos=None), dict(slots=None), dict(out=None), dict(qs=250), dict(ks=64), dict(vs=130), dict(k=P + 4), dict(os=252), dict(out=P, os=512),
                                 dict(out=2 * P), dict(out=3 * P)], ids=str)
def test_heads_refuse(ssd, bad):
    refused(ssd, heads(ssd, **bad), "ssd_norm_rope_kv")


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=P + 8), dict(dtype=0), dict(head_dim=96), dict(page_size=24), dict(pos_stride=32)], ids=str)
def test_heads_refuse_bad_caches(ssd, bad):
    refused(ssd, heads(ssd, pages(ssd, **bad)), "ssd_norm_rope_kv")


def test_heads_refuse_bad_norms_and_axes(ssd):
    for eps in (0.0, -1e-6, math.inf, math.nan):
        refused(ssd, heads(ssd, norm=ssd.ssd_head_norm(P, None, eps)), "ssd_norm_rope_kv")
    refused(ssd, heads(ssd, norm=ssd.ssd_head_norm(None, P + 4, 1e-6)), "ssd_norm_rope_kv")
    refused(ssd, heads(ssd, rp=ssd.ssd_rope_init(128)), "ssd_norm_rope_kv")
    axes = ssd.ssd_rope_axes_init(ssd.ssd_rope_init(64), ssd.SSD_AXES_SECTIONS, [16, 16])
    axes.axis[31] = 2
    refused(ssd, heads(ssd, axes=axes), "ssd_norm_rope_kv")
    refused(ssd, heads(ssd, axes=ssd.ssd_rope_axes()), "ssd_norm_rope_kv")
    assert heads(ssd, n_rows=0, q=None) == ssd.SSD_OK
    assert heads(ssd, n_rows=0, norm=ssd.ssd_head_norm(None, None, 0.0)) == ssd.SSD_OK  # (no gains: eps is not used)


@pytest.mark.parametrize("rot,pairs", [(128, [64]), (128, [16, 24, 24]), (64, [32, 0]), (48, [10, 7, 7]), (16, [2, 2, 2, 2]), (128, [24, 20, 20]), (32, [0, 16])])
@pytest.mark.parametrize("layout", [0, 1])
def test_axes(ssd, rot, pairs, layout):
    got = ssd.ssd_rope_axes_init(ssd.ssd_rope_init(rot), layout, pairs)
    want = ref.axis_of_pair(rot // 2, len(pairs), pairs, layout == 1)
    assert got.n_axes == len(pairs) and list(got.axis[:rot // 2]) == want and not any(got.axis[rot // 2:])


@pytest.mark.parametrize("layout,pairs", [(2, [32]), (0, []), (0, [8] * 5), (0, [31]), (0, [16, 17]), (1, [40, -8]), (0, [2**31 - 1, 33])], ids=str)
def test_axes_refuse(ssd, layout, pairs):
    with pytest.raises(ssd.SSDError) as e:
        ssd.ssd_rope_axes_init(ssd.ssd_rope_init(64), layout, pairs)
    assert e.value.code == ssd.SSD_ERR_INVALID_ARG and "ssd_rope_axes_init" in str(e.value)


# -- logits ----------------------------------------------------------------------

def rules(ssd, **kw):
    f = dict(vocab=1000, n_requests=2, n_rows=6, max_rows=3, row_start=P, history=P, history_len=P, prompt_len=None, history_stride=64, max_history=64,
             mask_words=1, tokens=P, masks=P, repetition=P, presence=None, frequency=None, bias=P, bias_of=None, allowed=P, allowed_of=P, bias_stride=1000,
             allowed_stride=32, n_bias=1, n_allowed=4)
    f.update(kw)
    assert list(f) == [x[0] for x in ssd.ssd_logit_rules._fields_]
    return ssd.ssd_logit_rules(*f.values())


def adjust(ssd, r=None, **kw):
    f = dict(dtype=ssd.SSD_F32, logits=2 * P, stride=1000, out=FAR, out_stride=1001, stream=None)
    f.update(kw)
    return ssd.lib.ssd_logits_adjust(r or rules(ssd), *f.values())


def choose(ssd, r=None, **kw):
    f = dict(dtype=ssd.SSD_BF16, logits=2 * P, stride=1000, k=4, tokens=FAR, logprob=2 * FAR, total=None, stream=None)
    f.update(kw)
    return ssd.lib.ssd_logits_choose(r or rules(ssd), *f.values())


BAD_RULES = [dict(vocab=0), dict(vocab=262145), dict(n_requests=0), dict(n_requests=4097), dict(n_rows=-1), dict(max_rows=0), dict(row_start=None), dict(history_len=None),
             dict(max_history=-1), dict(history_stride=63), dict(mask_words=0), dict(mask_words=5), dict(tokens=None), dict(masks=None), dict(bias_stride=999), dict(n_bias=0),
             dict(allowed_stride=31), dict(n_allowed=0), dict(allowed_of=None)]


@pytest.mark.parametrize("bad", BAD_RULES, ids=str)
def test_bad_rules_are_refused(ssd, bad):
    refused(ssd, adjust(ssd, rules(ssd, **bad)), "ssd_logits_adjust")
    refused(ssd, choose(ssd, rules(ssd, **bad)), "ssd_logits_choose")


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dtype=-1), dict(logits=None), dict(logits=P + 2), dict(stride=999), dict(out=None), dict(out=P + 1), dict(out_stride=999),
                                 dict(out=2 * P), dict(out=2 * P + 4, out_stride=1000), dict(out=2 * P + 4 * 5999, out_stride=1000)], ids=str)
def test_adjust_refuses(ssd, bad):
    refused(ssd, adjust(ssd, **bad), "ssd_logits_adjust")


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(logits=None), dict(logits=P + 1), dict(stride=999), dict(k=0), dict(k=17), dict(tokens=None), dict(logprob=None), dict(logprob=FAR),
                                 dict(total=FAR + 92), dict(tokens=P), dict(logprob=2 * P), dict(total=2 * P + 11996)], ids=str)
def test_choose_refuses(ssd, bad):
    refused(ssd, choose(ssd, **bad), "ssd_logits_choose")


def test_empty_logits_need_no_device(ssd):
    assert adjust(ssd, rules(ssd, n_rows=0), logits=None, out=None) == ssd.SSD_OK
    assert choose(ssd, rules(ssd, n_rows=0), logits=None, tokens=None) == ssd.SSD_OK
    assert ssd.lib.ssd_logits_choose(None, 0, P, 1000, 1, P, P, None, None) == ssd.SSD_ERR_INVALID_ARG


# -- mixture of experts ----------------------------------------------------------

def route(ssd, **kw):
    f = dict(dtype=ssd.SSD_BF16, n_rows=3, d=64, n_experts=8, k=2, x=P, xs=64, w=2 * P, favour=None, score=0, renorm=1, scale=1.0, ids=FAR, weights=2 * FAR, stream=None)
    f.update(kw)
    return ssd.lib.ssd_moe_route(*f.values())


@pytest.mark.parametrize("bad", [dict(dtype=0), dict(dtype=3), dict(n_rows=-1), dict(n_rows=65536), dict(d=0), dict(d=60), dict(d=65544), dict(n_experts=0), dict(n_experts=1025), dict(k=0),
                                 dict(k=17, n_experts=64), dict(k=9), dict(x=None), dict(x=P + 8), dict(xs=60), dict(xs=68), dict(w=None), dict(w=P + 8), dict(score=2), dict(renorm=2),
                                 dict(scale=math.inf), dict(scale=math.nan), dict(ids=None), dict(weights=None), dict(weights=FAR + 20), dict(ids=P)], ids=str)
def test_route_refuses(ssd, bad):
    refused(ssd, route(ssd, **bad), "ssd_moe_route")


def moe(ssd, **kw):
    f = dict(gate=P, up=P, down=P, gs=64 * 48, us=64 * 48, ds=64 * 48, dtype=ssd.SSD_BF16, n_experts=8, d=64, f=48)
    f.update(kw)
    return ssd.ssd_moe(*f.values())


def mlp(ssd, m=None, **kw):
    f = dict(n_rows=3, k=2, x=P, xs=64, ids=P, weights=P, residual=None, rs=0, out=FAR, os=64, ws=2 * FAR, wb=1 << 20, status=None, stream=None)
    f.update(kw)
    return ssd.lib.ssd_moe_mlp(m or moe(ssd), *f.values())


@pytest.mark.parametrize("bad", [dict(gate=None), dict(up=None), dict(down=None), dict(gate=P + 8), dict(down=P + 2), dict(gs=64 * 47), dict(us=64 * 48 + 4), dict(ds=0), dict(dtype=0),
                                 dict(n_experts=0), dict(n_experts=1025), dict(d=0), dict(d=68), dict(d=65544), dict(f=0), dict(f=44), dict(f=65544)], ids=str)
def test_bad_experts_are_refused(ssd, bad):
    refused(ssd, mlp(ssd, moe(ssd, **bad)), "ssd_moe_mlp")


@pytest.mark.parametrize("bad", [dict(n_rows=-1), dict(n_rows=1025), dict(k=0), dict(k=17), dict(x=None), dict(x=P + 8), dict(xs=56), dict(xs=68), dict(ids=None), dict(weights=None),
                                 dict(residual=P + 4, rs=64), dict(residual=P, rs=60), dict(residual=FAR, rs=72), dict(out=None), dict(out=P), dict(os=60), dict(ws=None),
                                 dict(ws=P + 8), dict(ws=FAR), dict(ids=FAR + 16), dict(x=2 * FAR + 64)], ids=str)
def test_mlp_refuses(ssd, bad):
    refused(ssd, mlp(ssd, **bad), "ssd_moe_mlp")


@pytest.mark.parametrize("bad", [dict(out=3 * FAR - 16), dict(ws=3 * FAR + 2 * 64 * 48 - 16), dict(status=3 * FAR + 2 * 64 * 48 * 8 - 4)], ids=str)
@pytest.mark.parametrize("which", ["gate", "up", "down"])
def test_mlp_refuses_results_in_its_matrices(ssd, which, bad):
    refused(ssd, mlp(ssd, moe(ssd, **{which: 3 * FAR}), **bad), "ssd_moe_mlp")


def test_mlp_says_when_the_workspace_is_short(ssd):
    n = ctypes.c_size_t()
    assert ssd.lib.ssd_moe_workspace(moe(ssd), 3, 2, n) == ssd.SSD_OK and n.value >= 2 * 2 * 6 * 48 + 4 * 6 * 64
    refused(ssd, mlp(ssd, wb=n.value - 1), "ssd_moe_mlp", ssd.SSD_ERR_CAPACITY)
    refused(ssd, ssd.lib.ssd_moe_workspace(moe(ssd), 3, 2, None), "ssd_moe_workspace")
    refused(ssd, ssd.lib.ssd_moe_workspace(moe(ssd, d=12), 3, 2, n), "ssd_moe_workspace")
    refused(ssd, ssd.lib.ssd_moe_workspace(moe(ssd), 1025, 2, n), "ssd_moe_workspace")


def test_empty_layers_need_no_device(ssd):
    assert route(ssd, n_rows=0, x=None) == ssd.SSD_OK
    assert mlp(ssd, n_rows=0, x=None, ws=None, wb=0) == ssd.SSD_OK


# -- addresses that the types do not have ------------------------------------------

@pytest.mark.parametrize("name", ["row_start", "history", "history_len", "prompt_len", "tokens", "masks", "repetition", "presence", "frequency", "bias", "bias_of", "allowed", "allowed_of"])
def test_unaligned_rules_are_refused(ssd, name):
    off = 4 if name == "masks" else 2
    for call in (adjust, choose):
        refused(ssd, call(ssd, rules(ssd, **{name: P + off})), "ssd_logits_adjust" if call is adjust else "ssd_logits_choose")
        assert b"aligned" in ssd.lib.ssd_last_error()


@pytest.mark.parametrize("bad", [dict(pos=P + 2), dict(slots=P + 1)], ids=str)
def test_unaligned_heads_are_refused(ssd, bad):
    refused(ssd, heads(ssd, **bad), "ssd_norm_rope_kv")
    assert b"aligned" in ssd.lib.ssd_last_error()


@pytest.mark.parametrize("bad", [dict(tokens=FAR + 2), dict(logprob=2 * FAR + 1), dict(total=3 * FAR + 2)], ids=str)
def test_unaligned_choices_are_refused(ssd, bad):
    refused(ssd, choose(ssd, **bad), "ssd_logits_choose")
    assert b"aligned" in ssd.lib.ssd_last_error()


@pytest.mark.parametrize("bad", [dict(ids=FAR + 2), dict(weights=2 * FAR + 2), dict(favour=P + 1)], ids=str)
def test_unaligned_routes_are_refused(ssd, bad):
    refused(ssd, route(ssd, **bad), "ssd_moe_route")
    assert b"aligned" in ssd.lib.ssd_last_error()


@pytest.mark.parametrize("bad", [dict(ids=P + 2), dict(weights=P + 2), dict(status=3 * FAR + 2)], ids=str)
def test_unaligned_layers_are_refused(ssd, bad):
    refused(ssd, mlp(ssd, **bad), "ssd_moe_mlp")
    assert b"aligned" in ssd.lib.ssd_last_error()


# -- what dependent launches keep to (a stale value or a hang otherwise) -------------

def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


@pytest.mark.parametrize("name", ["step_heads.cu", "step_logits.cu", "step_moe.cu", "step_ops.cuh"])
def test_no_non_coherent_loads(name):
    src = source(name)
    assert "global.nc" not in src and "__ldg(" not in src and "__restrict__" not in src


@pytest.mark.parametrize("name,kernels", [("step_heads.cu", ["heads_kernel"]), ("step_logits.cu", ["logits_kernel"]), ("step_moe.cu", ["route_kernel", "moe_up_kernel"])])
def test_kernels_wait_for_the_one_before(name, kernels):
    src = source(name)
    for k in kernels:
        body = src[re.search(r"\b%s\(const" % k, src).start():]
        body = body[:body.index("\n}\n")]
        before = body[:body.index("pdl_wait()")]
        assert "pdl_launch_dependents()" in body and "__ldcg" not in before and "return" not in before, k


def test_the_down_kernel_starts_when_ids_are_there():
    """It reads ids before it waits, so the kernel before it may only let it start once it has itself waited."""
    src = source("step_moe.cu")
    up = src[src.index("moe_up_kernel(const"):]
    assert 0 < up.index("pdl_wait()") < up.index("pdl_launch_dependents()")


# -- the oracle itself ------------------------------------------------------------

def test_reference_rules_by_hand():
    r = dict(history=np.array([[1, 1, 2, 9, -1, 3]], np.int32), history_len=np.array([5]), prompt_len=np.array([1]), tokens=np.array([4, 2], np.int32),
             masks=np.array([[1], [3]], np.int64), repetition=np.array([2.0], np.float32), presence=np.array([0.25], np.float32), frequency=np.array([0.5], np.float32),
             bias=np.array([[0, 0, 0, 0, 0, 8]], np.float32), allowed=np.array([[0b111110]], np.int32), allowed_of=np.array([0, -1]))
    x = np.array([5, 4, -4, 3, 2, 1], np.float32)
    # token 1: in the prompt and said once; 2: said once, and once more by node 1; 4: node 0; 9 and -1 are none
    assert ref.adjusted(x, 6, 0, 0, 0, 0, 2, r).tolist() == [-math.inf, 1.25, -8.75, 3.0, 0.25, 9.0]
    assert ref.adjusted(x, 6, 0, 1, 1, 0, 2, r).tolist() == [5.0, 1.25, -9.25, 3.0, 0.25, 9.0]
    assert ref.chosen(np.array([1, 3, 3, -np.inf, np.nan]), 4)[0] == [1, 2, 0, -1]
    assert ref.chosen(np.array([np.inf, 0, np.inf]), 3)[1] == [-math.log(2), -math.log(2), -math.inf]
