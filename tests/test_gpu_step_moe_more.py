"""ssd_moe_route and ssd_moe_mlp on the GPU: how exact the activations are, workspaces, waits that give up, NaN and infinities.  Plain numpy in 64 bits."""
import numpy as np
import pytest

import test_gpu_step_moe as moe

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ssd():
    import paper_2309_08168_gb300 as m
    return m


def differences(ssd, typ, n, scale, gain):
    """The activations of expert 0's units 2i and 2i + 1 are nearly alike, and output i is gain times their difference: what is
    lost of an activation on its way to the second product shows.  Returns (outputs, wanted ones, limits)."""
    t, half, d, f = moe.TYPES[typ], moe.HALF[typ], 64, 128
    g = torch.Generator().manual_seed(n)
    a = (0.5 + 3.0 * torch.rand(d, generator=g)).to(t).double()
    delta = (a * 2.0**-12 * torch.rand(d, generator=g).double()).to(t).double()
    x, gate, up, down = torch.zeros(n, d), torch.zeros(1, f, d), torch.zeros(1, f, d), torch.zeros(1, d, f)
    x[:, 0] = x[:, 1] = 2.0 ** -(torch.arange(n) % 2).float()
    gate[0, 0::2, 0], gate[0, 1::2, 0], gate[0, 1::2, 1] = a.float(), a.float(), delta.float()
    up[0, :, 0] = scale
    i = torch.arange(d)
    down[0, i, 2 * i], down[0, i, 2 * i + 1] = gain, -gain
    dev = [v.to(t).cuda() for v in (x, gate, up, down)]
    experts, out = ssd.MoeWeights(*dev[1:]), torch.empty(n, d, dtype=t, device="cuda")
    ids, weights = torch.zeros(n, 1, dtype=torch.int32, device="cuda"), torch.ones(n, 1, device="cuda")
    ws = torch.empty(ssd.ssd_moe_workspace(experts, n, 1), dtype=torch.uint8, device="cuda")
    ssd.ssd_moe_mlp(experts, dev[0], ids, weights, out, ws, cuda_stream=moe.stream())
    torch.cuda.synchronize()
    c = x[:, :1].double().numpy()
    h = [(lambda v: v / (1 + np.exp(-v)) * scale * c)(c * v.numpy()) for v in (a, a + delta)]
    want = gain * (h[0] - h[1])
    # an activation: products of few bits, exact; exp 2^-22 (two steps), 1 + exp, the division, the product with up and the weight 2^-24 each,
    # its values of the type 2^-22, and two sums of the matrix instructions, which cut off, 2^-22 each
    lim = 5 * 2.0**-22 * gain * (np.abs(h[0]) + np.abs(h[1])) + half * np.abs(want)
    return moe.f64(out), want, lim


@pytest.mark.parametrize("n", [1, 12, 40])
@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_activations_keep_their_bits(ssd, typ, n):
    got, want, lim = differences(ssd, typ, n, 1.0, 1.0)
    assert (np.abs(got - want) <= lim + 2.0**-25).all(), (np.abs(got - want) / lim).max()


@pytest.mark.parametrize("n", [1, 12, 40])
@pytest.mark.parametrize("scale", [2.0**-12, 2.0**-16])
@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_small_activations_keep_their_bits(ssd, typ, scale, n):
    """Activations near and below the lowest normal number of fp16, brought back by large weights: off by 2^-36 where that is more than
    2^-22 of them."""
    gain = 2.0**12
    got, want, lim = differences(ssd, typ, n, scale, gain)
    assert (np.abs(got - want) <= lim + 2 * gain * 2.0**-36 + 2.0**-25).all(), (np.abs(got - want) / lim).max()


def test_a_workspace_for_the_largest_round(ssd):
    """Seven rows have their sums over f in two parts, eight in one: the buffer for eight does for seven, and nothing behind it is written."""
    layers = [moe.Layer(ssd, 60, "bf16", n, 8192, 2048, 8, 1) for n in (8, 7)]
    size = ssd.ssd_moe_workspace(layers[0].experts, 8, 1)
    ws = torch.full((size + 4096,), 201, dtype=torch.uint8, device="cuda")
    for x in layers:
        x.ws = ws[:size]
        x.run()
        x.check([0, 6])
    assert (ws[size:] == 201).all()


@pytest.mark.parametrize("n,k,e", [(5, 3, 6), (20, 2, 4), (70, 1, 2)])
@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_a_wait_that_gives_up_leaves_nan(ssd, typ, n, k, e):
    """Without `status` too: a row is NaN where it misses something, or right; and the call after it is right."""
    x = moe.Layer(ssd, 12, typ, n, 512, 264, e, k)
    ssd.ssd_debug_moe_stall(1, 0.01)
    x.run()
    torch.cuda.synchronize()
    bad = torch.isnan(x.out[:, :512])
    rows = bad.any(1)
    assert rows.any() and torch.equal(bad.all(1), rows)  # (the second product's sums run over all that the first missed)
    x.check([r for r in range(n) if not rows[r]])
    x.run()
    x.check(range(0, n, 7))


def routed(z, k, favour, sigmoid, renorm):
    """(ids, weights) of one row's products z: NaN comes last and has no part in sums, +inf takes all of a softmax."""
    with np.errstate(all="ignore"):
        if sigmoid:
            p = 1.0 / (1.0 + np.exp(-z))
        else:
            p = np.where(z == np.nanmax(z), 1.0, np.exp(z - np.nanmax(z)))
            p = p / np.nansum(p)
        score = z if favour is None else p + favour  # (without favour the order of p is that of z)
        ids = sorted(range(len(z)), key=lambda e: (bool(np.isnan(score[e])), -score[e] if score[e] == score[e] else 0.0, e))[:k]
        q = p[ids]
        return ids, q / np.nansum(q) if renorm else q


@pytest.mark.parametrize("typ", ["f16", "bf16"])
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("favour", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("k,e", [(1, 9), (3, 9), (8, 9), (9, 9), (4, 300)])
def test_route_has_one_rule_for_nan_and_infinities(ssd, typ, score, favour, renorm, k, e):
    nan, inf = float("nan"), float("inf")
    head = [[0.5, nan, -1.5, 2.0, -0.25, 1.0, 0.5, nan, -2.0],       # NaN among ordinary products
            [0.5, inf, -1.5, 2.0, -0.25, inf, 0.5, nan, -inf],       # both infinities
            [-inf, -1.0, nan, -inf, 0.75, 3.0, -0.5, 0.0, 1.0],
            [nan, nan, nan, nan, nan, nan, nan, 1.0, nan]]           # one that is left
    z = torch.full((len(head), e), -6.0)
    z[:, :9] = torch.tensor(head)
    x, w = torch.zeros(len(head), 8 * len(head)), torch.zeros(len(head), e, 8 * len(head))
    f = torch.arange(e).float() % 7 / 16 if favour else None
    for r in range(len(head)):
        x[r, 8 * r] = 1.0
        w[r, :, 8 * r] = z[r]
        ids, weights = torch.full((1, k), -7, dtype=torch.int32, device="cuda"), torch.zeros(1, k, device="cuda")
        ssd.ssd_moe_route(x[r:r + 1].to(moe.TYPES[typ]).cuda(), w[r].to(moe.TYPES[typ]).cuda(), ids, weights, score=score, favour=None if f is None else f.cuda(), renorm=renorm,
                          cuda_stream=moe.stream())
        torch.cuda.synchronize()
        want, p = routed(z[r].double().numpy(), k, None if f is None else f.double().numpy(), score == 1, renorm)
        assert ids[0].tolist() == want, r
        np.testing.assert_allclose(moe.f64(weights)[0], p, rtol=16 * 2.0**-24, atol=2.0**-140, equal_nan=True)


@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_as_many_pairs_as_columns_in_registers_take(ssd, typ):
    """512 rows, 8 of 1024 experts each: the longest lists of pairs that go with eight columns a group."""
    x = moe.Layer(ssd, 61, typ, 512, 64, 520, 1024, 8)
    x.run()
    x.check([0, 1, 255, 511])


@pytest.mark.parametrize("typ", ["f16", "bf16"])
@pytest.mark.parametrize("n", [20, 40, 100])
def test_copied_columns_with_f_in_parts(ssd, typ, n):
    """16 and 32 columns a group, and sums over f in two parts."""
    x = moe.Layer(ssd, 62, typ, n, 64, 4104, 4, 2)
    x.run()
    x.check(range(0, n, 9))
