"""ssd_norm_rope_kv on the GPU: axes in turns with halves, and rounds of many rows of few heads.  Plain numpy in 64 bits."""
import pytest

import test_gpu_step_heads as heads

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ssd():
    import paper_2309_08168_gb300 as m
    return m


@pytest.mark.parametrize("c", [
    dict(typ="bf16", n=9, heads=8, kv_heads=2, hd=128, rot=128, interleaved=False, pairs=[24, 20, 20], in_turns=True),
    dict(typ="f16", n=5, heads=3, kv_heads=3, hd=64, rot=48, interleaved=False, pairs=[8, 8, 8], in_turns=True, layout="pos"),
    dict(typ="f32", n=6, heads=5, kv_heads=1, hd=128, rot=64, interleaved=False, pairs=[20, 4, 4, 4], in_turns=True, norm="q", packed=False),
], ids=lambda c: "-".join(str(v) for v in c.values()))
def test_axes_in_turns_with_halves(ssd, c):
    x = heads.Case(ssd, 70, **c)
    before = (x.kc.cpu(), x.vc.cpu())
    x.run()
    torch.cuda.synchronize()
    x.check(before)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("interleaved,hd,rot", [(False, 64, 64), (True, 128, 48)])
def test_many_rows_of_few_heads(ssd, typ, interleaved, hd, rot):
    """2500 rows of 4 + 1 heads: a row's CTA has half as many threads.  All rows equal those of small rounds, which the reference checks."""
    x, y = (heads.Case(ssd, 71, typ, 2500, 4, 1, hd, rot, interleaved, pairs=[rot // 2 - 6, 4, 2], page=48) for _ in range(2))
    x.run()
    pos, slots = y.positions.cuda(), y.slots.cuda()
    for r in range(0, 2500, 500):
        s = slice(r, r + 500)
        ssd.ssd_norm_rope_kv(y.kv, 1, y.rope, y.q[s], y.k[s], y.v[s], pos[:, s].contiguous(), slots[s].contiguous(), y.out[s], axes=y.axes, norm=y.norm, cuda_stream=heads.stream())
    torch.cuda.synchronize()
    assert torch.equal(x.out, y.out) and torch.equal(x.kc, y.kc) and torch.equal(x.vc, y.vc)
    out = x.out.double().cpu().numpy()
    half = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}[x.t]
    for r in (0, 1, 2, 1249, 2499):
        want, err = x.expected("q", r)
        assert (abs(out[r] - want) <= err + half * (abs(want) + err) + 2.0**-25).all(), r
