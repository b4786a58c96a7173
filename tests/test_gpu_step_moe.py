"""ssd_moe_route and ssd_moe_mlp on the GPU against plain numpy in 64 bits (tests/step_reference.py).

Experts are equal; weights are off by at most 16 roundings of fp32 (two of exp, five levels of a sum, the division, the scale).
"""
import numpy as np
import pytest

import step_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f16": 2.0**-11, "bf16": 2.0**-8}


@pytest.fixture(scope="module")
def ssd():
    import paper_2309_08168_gb300 as m
    return m


def stream():
    return torch.cuda.current_stream().cuda_stream


def f64(t):
    return t.double().cpu().numpy()


# -- route ------------------------------------------------------------------------

@pytest.mark.parametrize("typ", ["f16", "bf16"])
@pytest.mark.parametrize("n,d,e,k", [(1, 8, 1, 1), (2, 64, 2, 2), (5, 1000, 7, 3), (1, 4096, 8, 2), (9, 2048, 128, 8), (3, 520, 60, 16), (33, 264, 257, 6), (2, 136, 1024, 16), (300, 40, 9, 2)])
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("favour,renorm,scale", [(False, True, 1.0), (True, False, 2.5), (True, True, 1.0), (False, False, 0.5)])
def test_route(ssd, typ, n, d, e, k, score, favour, renorm, scale):
    g = torch.Generator().manual_seed(n * 1000 + e)
    x, w = torch.randn(n, d + 8, generator=g).to(TYPES[typ]).cuda()[:, :d], (torch.randn(e, d, generator=g) / d**0.5).to(TYPES[typ]).cuda()
    bias = (0.2 * torch.randn(e, generator=g)).cuda() if favour else None
    ids, weights = torch.full((n, k), -7, dtype=torch.int32, device="cuda"), torch.zeros(n, k, device="cuda")
    ssd.ssd_moe_route(x, w, ids, weights, score=score, favour=bias, renorm=renorm, scale=scale, cuda_stream=stream())
    torch.cuda.synchronize()
    want, p = ref.routed(f64(x), f64(w), k, None if bias is None else bias.cpu().numpy(), score == 1, renorm, scale)
    assert np.array_equal(ids.cpu().numpy(), want)
    np.testing.assert_allclose(f64(weights), p, rtol=16 * 2.0**-24, atol=2.0**-140)


def test_route_tells_close_experts_apart(ssd):
    """Scores whose difference is under a rounding of fp32 sums: exact sums order them, and equal ones go to the lowest."""
    d, e = 4096, 64
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn(4, d, generator=g).to(torch.bfloat16).cuda(), torch.empty(e, d, dtype=torch.bfloat16, device="cuda")
    w[:] = (torch.randn(d, generator=g) * 4).to(torch.bfloat16).cuda()
    for i in range(e):
        w[i, 7] = 2.0**-30 * (i % 32)  # the rest is the same sum
    ids, weights = torch.empty(4, 16, dtype=torch.int32, device="cuda"), torch.empty(4, 16, device="cuda")
    ssd.ssd_moe_route(x, w, ids, weights, cuda_stream=stream())
    torch.cuda.synchronize()
    for r in range(4):
        up = float(x[r, 7]) > 0
        order = sorted(range(e), key=lambda i: ((-(i % 32) if up else i % 32), i))
        assert ids[r].tolist() == order[:16]


def test_route_with_nan_and_infinities(ssd):
    x, w = torch.ones(2, 64, dtype=torch.float16, device="cuda"), torch.zeros(5, 64, dtype=torch.float16, device="cuda")
    w[1], w[2, 3], w[3] = 0.5, float("nan"), -float("inf")
    ids, weights = torch.empty(2, 5, dtype=torch.int32, device="cuda"), torch.empty(2, 5, device="cuda")
    ssd.ssd_moe_route(x, w, ids, weights, score=ssd.SSD_MOE_SIGMOID, renorm=False, cuda_stream=stream())
    torch.cuda.synchronize()
    assert ids.tolist() == [[1, 0, 4, 3, 2]] * 2
    p = weights[0].tolist()
    assert abs(p[0] - 1) < 1e-7 and p[1] == p[2] == 0.5 and p[3] == 0.0 and p[4] != p[4]


@pytest.mark.parametrize("score,favour", [(0, True), (1, False), (1, True)])
def test_route_of_scores_below_fp32(ssd, score, favour):
    """Products from -400 to 0: renormalised weights are ratios, however small the scores.  (Sums of few powers of two: the products are exact.)"""
    n, e, k = 6, 24, 4
    x, w = torch.zeros(n, 8, dtype=torch.bfloat16), torch.zeros(e, 8, dtype=torch.bfloat16)
    x[:, 0], x[:, 1] = 1.0, torch.tensor([0.0, -8.0, -20.0, -40.0, -50.0, 1.0])
    w[:, 0], w[:, 1] = -torch.arange(e) / 4.0, 8.0
    w[0] = 0.0
    bias = torch.zeros(e)
    bias[5:12] = torch.arange(7) * 0.25 + 2.0  # (these come first)
    if not favour:
        w[0, 0], w[0, 1] = -3.0, 8.0
    x, w, bias = x.cuda(), w.cuda(), bias.cuda() if favour else None
    ids, weights = torch.empty(n, k, dtype=torch.int32, device="cuda"), torch.empty(n, k, device="cuda")
    for renorm in (True, False):
        ssd.ssd_moe_route(x, w, ids, weights, score=score, favour=bias, renorm=renorm, cuda_stream=stream())
        torch.cuda.synchronize()
        want, p = ref.routed(f64(x), f64(w), k, None if bias is None else bias.cpu().numpy(), score == 1, renorm, 1.0)
        assert np.array_equal(ids.cpu().numpy(), want)
        np.testing.assert_allclose(f64(weights), p, rtol=16 * 2.0**-24, atol=2.0**-140)


# -- products ---------------------------------------------------------------------

class Layer:
    def __init__(self, ssd, seed, typ, n, d, f, e, k, residual=True, fused=False, pad=0, x_scale=1.0, ids=None):
        g = torch.Generator().manual_seed(seed)
        t, self.typ, self.ssd = TYPES[typ], typ, ssd

        def normal(*shape, std):
            return (std * torch.randn(*shape, generator=g)).to(t).cuda()
        self.x = normal(n, d + pad, std=x_scale)[:, :d]
        if fused:  # gate and up of an expert behind one another
            both = normal(e, 2, f, d, std=d**-0.5)
            self.gate, self.up = both[:, 0], both[:, 1]
        else:
            self.gate, self.up = normal(e, f, d, std=d**-0.5), normal(e, f, d, std=d**-0.5)
        self.down = normal(e, d, f, std=f**-0.5)
        self.residual = normal(n, d + pad, std=1.0)[:, :d] if residual else None
        self.ids = ids if ids is not None else torch.stack([torch.randperm(max(e, k), generator=g)[:k] for _ in range(n)]).int() if n else torch.empty(0, k, dtype=torch.int32)
        self.ids = self.ids.cuda()
        self.weights = torch.rand(n, k, generator=g).cuda()
        self.experts = ssd.MoeWeights(self.gate, self.up, self.down)
        self.out = torch.full((n, d + 8), 7.0, dtype=t, device="cuda")
        self.ws = torch.full((ssd.ssd_moe_workspace(self.experts, n, k),), 255, dtype=torch.uint8, device="cuda")
        self.d = d

    def run(self, out=None, residual=True):
        self.ssd.ssd_moe_mlp(self.experts, self.x, self.ids, self.weights, self.out[:, :self.d] if out is None else out, self.ws, residual=self.residual, cuda_stream=stream())

    def check(self, rows=None):
        torch.cuda.synchronize()
        rows = range(self.x.shape[0]) if rows is None else rows
        for r in rows:
            s = slice(r, r + 1)
            want, err = ref.mlp(f64(self.x[s]), self.ids[s].cpu().numpy(), self.weights[s].cpu().numpy(), Lazy(self.gate), Lazy(self.up), Lazy(self.down),
                                None if self.residual is None else f64(self.residual[s]), HALF[self.typ])
            got = f64(self.out[s, :self.d])
            lim = err + HALF[self.typ] * (np.abs(want) + err) + 2.0**-25
            assert (np.abs(got - want) <= lim).all(), (r, np.abs(got - want).max(), (np.abs(got - want) / lim).max())
        assert (self.out[:, self.d:] == 7.0).all()


class Lazy:
    """An expert's matrix in 64 bits when it is asked for."""

    def __init__(self, t):
        self.t, self.shape = t, tuple(t.shape)

    def __getitem__(self, e):
        return f64(self.t[e])


CASES = [
    dict(n=1, d=8, f=8, e=1, k=1),
    dict(n=1, d=264, f=88, e=4, k=2),
    dict(n=3, d=1024, f=2056, e=5, k=3, residual=False),
    dict(n=8, d=136, f=72, e=3, k=2),
    dict(n=9, d=136, f=72, e=3, k=2),
    dict(n=33, d=264, f=120, e=2, k=1, pad=8),
    dict(n=64, d=520, f=264, e=16, k=4, fused=True),
    dict(n=70, d=72, f=40, e=1, k=1),
    dict(n=13, d=48, f=1000, e=300, k=8),
    dict(n=200, d=64, f=48, e=9, k=16, residual=False),
    dict(n=1024, d=16, f=16, e=1024, k=16),
    dict(n=17, d=2048, f=768, e=8, k=2),
]


@pytest.mark.parametrize("typ", ["f16", "bf16"])
@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_mlp(ssd, typ, c):
    x = Layer(ssd, 3, typ, **c)
    x.run()
    x.check(None if x.x.shape[0] <= 64 else [0, 1, 31, 32, 63, 64, x.x.shape[0] - 1])


@pytest.mark.parametrize("n", [1, 7, 40])
def test_slots_that_go_nowhere_and_experts_twice(ssd, n):
    g = torch.Generator().manual_seed(n)
    ids = torch.randint(-2, 7, (n, 6), generator=g).int()
    ids[:, 3] = ids[:, 2]
    if n > 2:
        ids[1] = -1            # a row without experts
        ids[2] = 3             # one expert in all slots
    x = Layer(ssd, 5, "bf16", n, 96, 200, 5, 6, ids=ids)
    x.run()
    x.check()


@pytest.mark.parametrize("residual", [True, False])
def test_no_expert_at_all(ssd, residual):
    x = Layer(ssd, 5, "f16", 4, 72, 40, 5, 2, ids=torch.full((4, 2), 5, dtype=torch.int32), residual=residual)
    x.run()
    torch.cuda.synchronize()
    assert torch.equal(x.out[:, :72], x.residual if residual else torch.zeros_like(x.x))


def test_one_expert_for_all(ssd):
    """Eight rows of one expert twice each (two groups of a small batch), and 100 of one (four of a large one)."""
    for n, k in ((8, 2), (100, 1)):
        x = Layer(ssd, 6, "bf16", n, 256, 320, 3, k, ids=torch.full((n, k), 1, dtype=torch.int32))
        x.run()
        x.check()


def test_small_values(ssd):
    x = Layer(ssd, 8, "f16", 5, 256, 256, 4, 2, residual=False, x_scale=0.02)
    x.run()
    x.check()


def test_infinities_stay_in_their_rows(ssd):
    x, y = (Layer(ssd, 9, "bf16", 12, 256, 264, 4, 2) for _ in range(2))
    y.x[5, 77], y.x[6, 0] = float("inf"), float("nan")
    x.run()
    y.run()
    torch.cuda.synchronize()
    keep = [r for r in range(12) if r not in (5, 6)]
    assert torch.equal(x.out[keep], y.out[keep])
    assert not torch.isfinite(y.out[5, :256]).any() and torch.isnan(y.out[6, :256]).all()


def test_in_the_residuals_place_and_the_same_bits_again(ssd):
    x = Layer(ssd, 10, "f16", 20, 512, 264, 8, 4)
    x.run()
    torch.cuda.synchronize()
    first = x.out[:, :512].clone()
    for _ in range(5):
        x.run()
        torch.cuda.synchronize()
        assert torch.equal(first, x.out[:, :512])
    y = x.residual.clone()
    ssd.ssd_moe_mlp(x.experts, x.x, x.ids, x.weights, y, x.ws, residual=y, cuda_stream=stream())
    torch.cuda.synchronize()
    assert torch.equal(first, y)


def test_layers_behind_one_another_and_replayed(ssd):
    """Router and products of four layers through one workspace, eager and captured, with ids that change from layer to layer."""
    n, d, f, e, k = 6, 256, 136, 16, 4
    layers = [Layer(ssd, 30 + i, "bf16", n, d, f, e, k) for i in range(4)]
    routers = [(torch.randn(e, d, generator=torch.Generator().manual_seed(i)) / 16).to(torch.bfloat16).cuda() for i in range(4)]
    ids, w, ws = layers[0].ids, layers[0].weights, layers[0].ws
    start = layers[0].x.contiguous()
    bufs = [torch.empty_like(start) for _ in range(5)]

    def forward(s):
        bufs[0].copy_(start)
        for i in range(4):
            ssd.ssd_moe_route(bufs[i], routers[i], ids, w, cuda_stream=s)
            ssd.ssd_moe_mlp(layers[i].experts, bufs[i], ids, w, bufs[i + 1], ws, residual=bufs[i], cuda_stream=s)
    forward(stream())
    torch.cuda.synchronize()
    want = [b.clone() for b in bufs]
    # each layer alone, waited for
    for i in range(4):
        ssd.ssd_moe_route(want[i], routers[i], ids, w, cuda_stream=stream())
        torch.cuda.synchronize()
        out = torch.empty_like(start)
        ssd.ssd_moe_mlp(layers[i].experts, want[i], ids, w, out, ws, residual=want[i], cuda_stream=stream())
        torch.cuda.synchronize()
        assert torch.equal(out, want[i + 1]), i
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        forward(torch.cuda.current_stream().cuda_stream)
    for b in bufs:
        b.zero_()
    for _ in range(20):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(bufs, want))


def test_two_layers_on_two_streams(ssd):
    xs = [Layer(ssd, 40 + i, "bf16", 9 + 20 * i, 512, 264, 16, 4) for i in range(2)]
    for x in xs:
        x.run()
    torch.cuda.synchronize()
    want = [x.out.clone() for x in xs]
    outs = [[torch.zeros_like(x.out) for _ in range(8)] for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for i in range(8):
        for x, o, s in zip(xs, outs, streams):
            ssd.ssd_moe_mlp(x.experts, x.x, x.ids, x.weights, o[i][:, :512], x.ws, residual=x.residual, cuda_stream=s.cuda_stream)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(w[:, :512], y[:, :512]) for y in o)


def test_experts_beyond_32_bits(ssd):
    """Experts and rows whose offsets pass 2^31 elements."""
    d, f, e, n, far = 64, 40, 3, 3, (1 << 31) + 64
    big = torch.zeros(2 * far + 4 * d * f, dtype=torch.bfloat16, device="cuda")
    x = Layer(ssd, 50, "bf16", n, d, f, e, 3)
    size = d * f
    gate, up = (torch.as_strided(big, (e, f, d), (far, d, 1), i * size) for i in (0, 1))
    down, rows = torch.as_strided(big, (e, d, f), (far, f, 1), 2 * size), torch.as_strided(big, (n, d), (far, 1), 3 * size)
    for a, b in ((gate, x.gate), (up, x.up), (down, x.down), (rows, x.x)):
        a.copy_(b)
    x.run()
    torch.cuda.synchronize()
    want = x.out.clone()
    x.gate, x.up, x.down, x.x = gate, up, down, rows
    x.experts = ssd.MoeWeights(gate, up, down)
    x.out.fill_(7.0)
    x.run()
    torch.cuda.synchronize()
    assert torch.equal(x.out, want)
    ids, weights = x.ids.clone(), x.weights.clone()
    for r in (rows, rows.contiguous()):
        ssd.ssd_moe_route(r, x.gate[0].contiguous(), ids, weights, cuda_stream=stream())
        torch.cuda.synchronize()
        if r is rows:
            first = ids.clone(), weights.clone()
    assert torch.equal(first[0], ids) and torch.equal(first[1], weights)


def test_a_wait_that_gives_up_is_told(ssd):
    x = Layer(ssd, 12, "bf16", 5, 512, 264, 6, 3)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ssd.ssd_debug_moe_stall(1, 0.01)
    ssd.ssd_moe_mlp(x.experts, x.x, x.ids, x.weights, x.out[:, :512], x.ws, residual=x.residual, status=status, cuda_stream=stream())
    torch.cuda.synchronize()
    assert status.item() == ssd.SSD_STATUS_TIMEOUT
    status.zero_()
    ssd.ssd_debug_moe_stall(1, 0.01)
    ssd.ssd_debug_moe_stall(-1)
    ssd.ssd_moe_mlp(x.experts, x.x, x.ids, x.weights, x.out[:, :512], x.ws, residual=x.residual, status=status, cuda_stream=stream())
    x.check()
    assert status.item() == 0
    for bad in (0.0, 11.0):
        with pytest.raises(ssd.SSDError):
            ssd.ssd_debug_moe_stall(0, bad)


def test_the_binding_refuses(ssd):
    x = Layer(ssd, 1, "f16", 3, 64, 40, 4, 2)
    for bad in (dict(x=x.x[:, :56]), dict(x=x.x.bfloat16()), dict(ids=x.ids.long()), dict(ids=x.ids[:2]), dict(weights=x.weights.half()), dict(out=x.out), dict(ws=x.ws[:-1]),
                dict(ws=x.ws.int()), dict(x=x.x.cpu()), dict(residual=x.residual[:2])):
        a = {"x": x.x, "ids": x.ids, "weights": x.weights, "out": x.out[:, :64], "ws": x.ws, "residual": None, **bad}
        with pytest.raises(ssd.SSDError):
            ssd.ssd_moe_mlp(x.experts, a["x"], a["ids"], a["weights"], a["out"], a["ws"], residual=a["residual"])
    for bad in ((x.gate, x.up, x.up), (x.gate, x.up[:3], x.down), (x.gate, x.up.bfloat16(), x.down), (x.gate.float(), x.up.float(), x.down.float()),
                (x.gate.transpose(1, 2), x.up.transpose(1, 2), x.down.transpose(1, 2))):
        with pytest.raises(ssd.SSDError):
            ssd.MoeWeights(*bad)
    w = torch.zeros(4, 64, dtype=torch.float16, device="cuda")
    for bad in ((x.x.float(), w.float(), x.ids, x.weights), (x.x, w[:, :56], x.ids, x.weights), (x.x, w, x.ids.long(), x.weights), (x.x, w, x.ids, x.weights[:2])):
        with pytest.raises(ssd.SSDError):
            ssd.ssd_moe_route(*bad)
