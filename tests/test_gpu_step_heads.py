"""ssd_norm_rope_kv on the GPU against plain numpy in 64 bits (tests/step_reference.py)."""
import numpy as np
import pytest

import step_reference as ref
import tree_reference

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": (torch.float32, torch.float16), "f16": (torch.float16, torch.float16), "bf16": (torch.bfloat16, torch.bfloat16)}


@pytest.fixture(scope="module")
def ssd():
    import paper_2309_08168_gb300 as m
    return m


def stream():
    return torch.cuda.current_stream().cuda_stream


class Case:
    def __init__(self, ssd, seed, typ, n, heads, kv_heads, hd, rot, interleaved, pairs=None, in_turns=False, norm="both", page=16, layers=2, far=50000, amplitude=1.0,
                 layout="head", packed=True, scale=1.5):
        g = torch.Generator().manual_seed(seed)
        self.ssd, self.t, self.ct = ssd, *TYPES[typ]
        self.n, self.heads, self.kv_heads, self.hd, self.rot, self.inter, self.page, self.amp = n, heads, kv_heads, hd, rot, interleaved, page, amplitude
        self.pairs, self.in_turns = pairs, in_turns
        w = [heads * hd, kv_heads * hd, kv_heads * hd]
        all_ = (scale * torch.randn(n, sum(w) + (64 if packed else 0), generator=g)).to(self.t).cuda()
        parts = all_[:, :sum(w)].split(w, 1)
        if not packed:
            parts = [p.contiguous() for p in parts]
        self.q, self.k, self.v = (p.unflatten(1, (-1, hd)) for p in parts)
        pages = -(-n * 3 // 2 // page) + 1
        shape = {"head": (layers, pages, kv_heads, page, hd), "pos": (layers, pages, page, kv_heads, hd)}[layout]
        self.kc, self.vc = ((torch.randn(*shape, generator=g)).to(self.ct).cuda() for _ in range(2))
        if layout == "pos":
            self.kc, self.vc = self.kc.transpose(2, 3), self.vc.transpose(2, 3)
        self.slots = torch.randperm(pages * page, generator=g)[:n].int()
        if n > 2:
            self.slots[1], self.slots[2] = -1, pages * page  # no place, and one outside
        axes = len(pairs) if pairs else 1
        self.positions = torch.randint(-3, far, (axes, n), generator=g).int()
        self.gain = {x: (1 + 0.3 * torch.randn(hd, generator=g)).cuda() if norm in ("both", x) else None for x in "qk"}
        self.rope = ssd.ssd_rope_init(rot, theta=1e4, interleaved=interleaved, amplitude=amplitude)
        self.axes = ssd.ssd_rope_axes_init(self.rope, int(in_turns), pairs) if pairs else None
        self.kv = ssd.PagedKV(self.kc, self.vc)
        self.norm = ssd.HeadNorm(self.gain["q"], self.gain["k"], 1e-5) if norm != "none" else None
        self.out = torch.full((n, heads, hd), 7.0, dtype=self.t, device="cuda")

    def run(self, layer=1, out=None):
        self.ssd.ssd_norm_rope_kv(self.kv, layer, self.rope, self.q, self.k, self.v, self.positions.cuda(), self.slots.cuda(), self.out if out is None else out, axes=self.axes,
                                  norm=self.norm, cuda_stream=stream())

    def expected(self, name, row):
        axis = ref.axis_of_pair(self.rot // 2, len(self.pairs), self.pairs, self.in_turns) if self.pairs else [0] * (self.rot // 2)
        gain = None if self.gain[name] is None else self.gain[name].cpu().numpy()
        x = (self.q if name == "q" else self.k)[row].double().cpu().numpy()
        pos, rates = self.positions[:, row].tolist(), tree_reference.frequencies(self.rot, 1e4)
        y = ref.turned(x, gain, 1e-5, pos, axis, rates, self.rot, self.inter, self.amp)
        # what a result is made of: its pair's absolute values (20 roundings: 13 of the sum of squares halved, reciprocal root 4, angle and
        # sine 4, gain, products and sum 4)
        z = np.abs(ref.turned(x, gain, 1e-5, [0] * len(pos), axis, rates, self.rot, self.inter, self.amp))
        m = z.copy()
        for i in range(self.rot // 2):
            lo, hi = (2 * i, 2 * i + 1) if self.inter else (i, i + self.rot // 2)
            m[:, lo] = m[:, hi] = z[:, lo] + z[:, hi]
        return y, 20 * 2.0**-24 * m

    def check(self, before):
        out, kc, vc = self.out.double().cpu().numpy(), self.kc.cpu(), self.vc.cpu()
        want_k, want_v = (x.clone() for x in before)
        half = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}
        tiny = {torch.float32: 2.0**-149, torch.float16: 2.0**-25, torch.bfloat16: 2.0**-133}

        def near(got, want, err, t):
            assert (np.abs(got - want) <= err + half[t] * (np.abs(want) + err) + tiny[t]).all(), np.abs(got - want).max()
        for r in range(self.n):
            near(out[r], *self.expected("q", r), self.t)
            s = int(self.slots[r])
            if 0 <= s < self.kc.shape[1] * self.page:
                at = (1, s // self.page, slice(None), s % self.page)
                near(kc[at].double().numpy(), *self.expected("k", r), self.ct)
                want_k[at] = kc[at]
                want_v[at] = self.v[r].to(self.ct).cpu()
        # all other rows as they were, values copied
        assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


CASES = [
    dict(typ="f32", n=1, heads=4, kv_heads=4, hd=64, rot=64, interleaved=False),
    dict(typ="bf16", n=5, heads=16, kv_heads=2, hd=128, rot=128, interleaved=False, pairs=[16, 24, 24]),
    dict(typ="f16", n=7, heads=5, kv_heads=5, hd=128, rot=48, interleaved=False, pairs=[8, 8, 8], layout="pos"),
    dict(typ="f16", n=3, heads=6, kv_heads=3, hd=64, rot=32, interleaved=True, pairs=[6, 5, 5], in_turns=True),
    dict(typ="f32", n=9, heads=33, kv_heads=11, hd=128, rot=16, interleaved=True, pairs=[2, 2, 2, 2], packed=False),
    dict(typ="bf16", n=4, heads=1, kv_heads=1, hd=64, rot=48, interleaved=False, norm="q"),
    dict(typ="f32", n=4, heads=2, kv_heads=1, hd=128, rot=128, interleaved=False, norm="k", amplitude=1.25, pairs=[0, 64]),
    dict(typ="bf16", n=6, heads=8, kv_heads=8, hd=128, rot=64, interleaved=True, norm="none", pairs=[11, 11, 10], in_turns=True),
    dict(typ="f16", n=650, heads=3, kv_heads=1, hd=64, rot=64, interleaved=False, pairs=[12, 10, 10], page=48),
    dict(typ="bf16", n=2, heads=128, kv_heads=40, hd=128, rot=128, interleaved=False, pairs=[24, 20, 20]),
    dict(typ="f32", n=5, heads=8, kv_heads=2, hd=64, rot=64, interleaved=False, far=2**31 - 1),
    dict(typ="f32", n=5, heads=8, kv_heads=2, hd=64, rot=64, interleaved=False, scale=1e-4),
    dict(typ="bf16", n=5, heads=8, kv_heads=2, hd=128, rot=128, interleaved=False, scale=1e6, norm="both"),
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_heads(ssd, c):
    x = Case(ssd, 5, **c)
    before = (x.kc.cpu(), x.vc.cpu())
    x.run()
    torch.cuda.synchronize()
    x.check(before)


def test_without_norms_it_does_what_rope_kv_does(ssd):
    a, b = (Case(ssd, 9, "f16", 20, 8, 4, 128, 64, False, norm="none") for _ in range(2))
    a.run()
    ssd.ssd_rope_kv(b.kv, 1, b.rope, b.q, b.k, b.v, b.positions.cuda()[0], b.slots.cuda(), b.out, stream())
    torch.cuda.synchronize()
    # (the two add their products in another order: fp32 roundings apart before the last one)
    for x, y in ((a.out, b.out), (a.kc, b.kc), (a.vc, b.vc)):
        assert torch.allclose(x.float(), y.float(), rtol=2.0**-10, atol=1e-6)


def test_queries_in_place_and_replays(ssd):
    a, b = (Case(ssd, 11, "bf16", 30, 8, 4, 128, 128, False, pairs=[24, 20, 20]) for _ in range(2))
    pos, slots = b.positions.cuda(), b.slots.cuda()
    a.run()
    side = torch.cuda.Stream()
    keep = b.q.clone()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            b.q.copy_(keep)
            ssd.ssd_norm_rope_kv(b.kv, 1, b.rope, b.q, b.k, b.v, pos, slots, b.q, axes=b.axes, norm=b.norm, cuda_stream=torch.cuda.current_stream().cuda_stream)
        for _ in range(3):
            g.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.out, b.q) and torch.equal(a.kc, b.kc) and torch.equal(a.vc, b.vc)


def test_rows_that_hold_infinities_do_not_reach_others(ssd):
    a, b = (Case(ssd, 13, "f16", 8, 4, 2, 64, 48, False) for _ in range(2))
    b.q[3, 1, 60], b.k[4, 1, 2] = float("inf"), float("nan")
    a.run()
    b.run()
    torch.cuda.synchronize()
    same = torch.ones(8, 4, dtype=torch.bool)
    same[3, 1] = False
    assert torch.equal(a.out.cpu()[same], b.out.cpu()[same])
    s = int(b.slots[4])
    diff = (a.kc != b.kc).cpu()
    diff[1, s // 16, 1, s % 16] = False
    assert not diff.any()


def test_rows_and_cache_beyond_32_bits(ssd):
    """Rows 2^30 values apart, and a cache whose layers are."""
    far = 1 << 30
    a, b = (Case(ssd, 15, "bf16", 4, 2, 1, 64, 64, False, pairs=[12, 10, 10]) for _ in range(2))
    big = torch.zeros(3 * far + 4 * 64, dtype=torch.bfloat16, device="cuda")
    b.q, b.k, b.v = (torch.as_strided(big, (4, h, 64), (far, 64, 1), o) for h, o in ((2, 0), (1, 128), (1, 192)))
    for x, y in ((b.q, a.q), (b.k, a.k), (b.v, a.v)):
        x.copy_(y)
    pages = a.kc.shape[1]
    store = [torch.zeros(2 * far + pages * 1024, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    b.kc, b.vc = (torch.as_strided(s, (2, pages, 1, 16, 64), (2 * far, 1024, 1024, 64, 1)) for s in store)
    b.kc.copy_(a.kc)
    b.vc.copy_(a.vc)
    b.kv = ssd.PagedKV(b.kc, b.vc)
    a.run()
    b.run()
    torch.cuda.synchronize()
    assert torch.equal(a.out, b.out) and torch.equal(a.kc, b.kc) and torch.equal(a.vc, b.vc)


def test_the_binding_refuses(ssd):
    x = Case(ssd, 1, "f16", 4, 4, 2, 64, 64, False, pairs=[16, 16])
    pos, slots = x.positions.cuda(), x.slots.cuda()
    with pytest.raises(ssd.SSDError):  # one axis' positions for two axes
        ssd.ssd_norm_rope_kv(x.kv, 0, x.rope, x.q, x.k, x.v, pos[0], slots, x.out, axes=x.axes, norm=x.norm)
    with pytest.raises(ssd.SSDError):  # gains of another width
        ssd.ssd_norm_rope_kv(x.kv, 0, x.rope, x.q, x.k, x.v, pos, slots, x.out, axes=x.axes, norm=ssd.HeadNorm(torch.ones(128, device="cuda"), None, 1e-5))
    with pytest.raises(ssd.SSDError):
        ssd.HeadNorm(torch.ones(64), None, 1e-5)
    with pytest.raises(ssd.SSDError):
        ssd.HeadNorm(torch.ones(64, device="cuda", dtype=torch.float16), None, 1e-5)
