"""ssd_logits_adjust and ssd_logits_choose on the GPU against plain numpy (tests/step_reference.py).

Adjusted logits are equal (every step is one fp32 rounding on both sides), chosen tokens too.  Log probabilities: a weight is off by
at most 2^-22 + d 2^-23 for a logit d below the largest, which is at most 13 2^-23 of the sum (d is under 13 on average over the weights), a sum of at most 72
chunk values and 12 levels by 84 2^-24; the results by a rounding of the largest value in them.
"""
import numpy as np
import pytest

import step_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
LEFT = -7


@pytest.fixture(scope="module")
def ssd():
    import paper_2309_08168_gb300 as m
    return m


def stream():
    return torch.cuda.current_stream().cuda_stream


def gpu(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def tree_masks(rng, counts, words):
    out = []
    for n in counts:
        seen = []
        for i in range(n):
            p = -1 if i == 0 else int(rng.integers(max(0, i - 5), i))
            seen.append((1 << i) | (seen[p] if p >= 0 else 0))
            out.append([(seen[i] >> (64 * w)) & (2**64 - 1) for w in range(words)])
    return np.array(out, np.uint64).reshape(-1, words).view(np.int64)


class Case:
    """rows: the requests' row counts, or None: a row a request."""

    def __init__(self, seed, typ, vocab, rows, n=None, hist=0, prompt=True, tree=True, tokens=True, parts="rpf", bias=0, bias_of=True, masks=0, mask_of=True, pad=0, lead=0, spare=0,
                 few=None, spread=3.0):
        rng = np.random.default_rng(seed)
        self.vocab, self.typ = vocab, typ
        counts = rows if rows is not None else [1] * n
        B, n = len(counts), sum(counts) + spare
        self.start = np.concatenate([[lead], lead + np.cumsum(counts)]).astype(np.int32) if rows is not None else np.arange(n + 1, dtype=np.int32)
        n += lead
        self.n, few = n, few or vocab
        r = self.r = {}
        if hist:
            r["history"] = rng.integers(-2, few + 2, (B, hist)).astype(np.int32)
            r["history_len"] = rng.integers(-1, hist + 2, B).astype(np.int32)
            r["history_len"][0] = hist
            if prompt:
                r["prompt_len"] = (r["history_len"] // 2).astype(np.int32)
        if hist or tokens:
            if tokens:
                r["tokens"] = rng.integers(-1, few + 1, n).astype(np.int32)
                if tree and rows is not None:
                    words = (max(counts) + 63) // 64
                    r["masks"] = np.concatenate([np.full((lead, words), -1, np.int64), tree_masks(rng, counts, words), np.full((spare, words), -1, np.int64)])
            for key, name in (("r", "repetition"), ("p", "presence"), ("f", "frequency")):
                if key in parts:
                    r[name] = rng.uniform(0.5, 2.0, B).astype(np.float32)
        if bias:
            r["bias"] = np.where(rng.random((bias, vocab)) < 0.1, 5 * rng.standard_normal((bias, vocab)), 0).astype(np.float32)
            if bias_of:
                r["bias_of"] = rng.integers(-1, bias + 1, B).astype(np.int32)
        if masks:
            bits = rng.integers(0, 2**32, (masks, -(-vocab // 32)), dtype=np.uint64).astype(np.uint32)
            bits[0] = 0  # leaves nothing
            if masks > 1:
                bits[1] = 0
                bits[1, (vocab - 1) // 32] = np.uint32(1 << ((vocab - 1) % 32))  # leaves the last
            r["allowed"] = bits.view(np.int32)
            if mask_of:
                r["allowed_of"] = rng.integers(-1, masks + 1, n).astype(np.int32)
        t = TYPES[typ]
        x = torch.from_numpy(spread * rng.standard_normal((n, vocab + pad))).to(t)
        self.logits = x.cuda()[:, :vocab]
        self.host = self.logits.float().cpu().numpy()
        self.max_rows = max(counts)
        self.has_start = rows is not None

    def rules(self, ssd, **kw):
        return ssd.LogitRules(self.vocab, self.n, row_start=gpu(self.start) if self.has_start else None, max_rows=self.max_rows, **{k: gpu(v) for k, v in self.r.items()}, **kw)

    def rows(self):
        """(row, request, node, first row, rows) of the rows that a request owns."""
        for b in range(len(self.start) - 1):
            for i in range(self.start[b + 1] - self.start[b]):
                yield int(self.start[b]) + i, b, i, int(self.start[b]), int(self.start[b + 1] - self.start[b])

    def expected(self):
        want = np.full((self.n, self.vocab), np.nan, np.float32)
        for row, b, node, start, count in self.rows():
            want[row] = ref.adjusted(self.host[row], self.vocab, b, row, node, start, count, self.r)
        return want


def check(ssd, c, k=4, want_adjust=True):
    rules = c.rules(ssd)
    want = c.expected()
    owned = np.zeros(c.n, bool)
    for row, *_ in c.rows():
        owned[row] = True
    t = TYPES[c.typ]
    if want_adjust:
        out = torch.full((c.n, c.vocab + 3), float(LEFT), dtype=t, device="cuda")
        ssd.ssd_logits_adjust(rules, c.logits, out[:, :c.vocab], stream())
        torch.cuda.synchronize()
        exact = torch.from_numpy(want).to(t)
        got = out[:, :c.vocab].cpu()
        bad = got[owned].float().numpy() != exact[owned].float().numpy()
        bad &= ~(np.isnan(got[owned].float().numpy()) & np.isnan(exact[owned].float().numpy()))
        assert not bad.any(), (np.argwhere(bad)[:5], bad.sum())
        assert (got[~owned] == LEFT).all() and (out[:, c.vocab:] == LEFT).all()
    tokens = torch.full((c.n, k), LEFT, dtype=torch.int32, device="cuda")
    logprob = torch.full((c.n, k), float(LEFT), device="cuda")
    total = torch.full((c.n,), float(LEFT), device="cuda")
    ssd.ssd_logits_choose(rules, c.logits, tokens, logprob, total, stream())
    torch.cuda.synchronize()
    tok, lp, tot = tokens.cpu().numpy(), logprob.cpu().numpy(), total.cpu().numpy()
    for row in range(c.n):
        if not owned[row]:
            assert (tok[row] == LEFT).all() and (lp[row] == LEFT).all() and tot[row] == LEFT
            continue
        best, prob, whole = ref.chosen(want[row], k)
        assert tok[row].tolist() == best, (row, tok[row], best)
        top = abs(float(np.nanmax(np.where(np.isfinite(want[row]), np.abs(want[row]), 0))))
        tol = 2 * 2.0**-22 + 13 * 2.0**-23 + 84 * 2.0**-24 + 3 * 2.0**-24 * max(1.0, top)
        for a, b in zip([*lp[row], tot[row]], [*prob, whole]):
            assert a == b or abs(a - b) <= tol + 2.0**-23 * abs(b), (row, a, b)
    return tokens, logprob, total


CASES = [
    dict(typ="f32", vocab=1, rows=[1, 2], tokens=False),
    dict(typ="f32", vocab=5, rows=None, n=3, hist=4, masks=3, bias=2),
    dict(typ="f16", vocab=31, rows=[3, 0, 2], hist=20, masks=4),
    dict(typ="bf16", vocab=1000, rows=[5, 1, 9], hist=300, few=60, bias=3),
    dict(typ="f32", vocab=2048, rows=[70, 3], hist=100, few=200, masks=5, lead=2, spare=3),
    dict(typ="bf16", vocab=5001, rows=[200, 7], hist=50, few=100, pad=3),
    dict(typ="f16", vocab=4097, rows=[6, 6], tree=False, hist=700, few=500, prompt=False, pad=1),
    dict(typ="f32", vocab=8191, rows=[40], tree=False, tokens=True, few=30),
    dict(typ="f32", vocab=32001, rows=None, n=4, hist=1000, tokens=False, parts="r", bias=1, bias_of=False),
    dict(typ="bf16", vocab=50257, rows=[4, 4], hist=2000, few=3000, parts="pf", masks=6),
    dict(typ="f16", vocab=131075, rows=[2, 1], hist=500, bias=2, masks=3, mask_of=False),
    dict(typ="f32", vocab=262144, rows=[1, 2], hist=4000, parts="f", pad=5),
    dict(typ="bf16", vocab=262143, rows=[2], hist=10, bias=1),
    dict(typ="f32", vocab=700, rows=None, n=700, hist=30, few=50, masks=7),
    dict(typ="f16", vocab=2500, rows=[17] * 30, hist=30, few=50, masks=7),
    dict(typ="bf16", vocab=3001, rows=[256], tokens=True, few=100),
    dict(typ="f16", vocab=262144, rows=[2], hist=60000, bias=1, masks=3),  # more said tokens than a list has room for
    dict(typ="bf16", vocab=5000, rows=[3, 2], hist=9000, masks=4),  # (nearly) every token said
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(str(v)[:20] for v in c.values()))
def test_logits(ssd, c):
    c = dict(c)
    if c.get("mask_of") is False:
        c["masks"] = sum(c["rows"])
    check(ssd, Case(3, **c), k=16 if c["vocab"] in (5000, 262144) else min(16, 1 + c["vocab"] % 7))


@pytest.mark.parametrize("k", [1, 2, 3, 8, 16])
@pytest.mark.parametrize("vocab,n", [(9, 2), (4000, 3), (33000, 1), (33000, 400), (200000, 2)])
def test_the_k_best(ssd, k, vocab, n):
    check(ssd, Case(17 + k, "bf16", vocab, None, n=n, tokens=False), k, want_adjust=False)


@pytest.mark.parametrize("k", [1, 5, 16])
def test_ties_go_to_the_lowest(ssd, k):
    c = Case(1, "f16", 40000, [4], tokens=False)
    c.logits[0] = 0.0                          # all alike
    c.logits[1] = torch.arange(40000, device="cuda").half() // 8 % 50   # many of each
    c.logits[2] = -float("inf")
    c.logits[2, 39999], c.logits[2, 20000], c.logits[2, 7] = -60000.0, -0.0, 0.0
    c.logits[3] = float("nan")
    c.host = c.logits.float().cpu().numpy()
    check(ssd, c, k, want_adjust=False)


@pytest.mark.parametrize("k", [1, 4, 16])
@pytest.mark.parametrize("typ,vocab,pad", [("f32", 32000, 0), ("bf16", 50257, 0), ("f16", 131075, 2)])
def test_masks_that_leave_few(ssd, k, typ, vocab, pad):
    """Up to a 32nd of a slice, where only the tokens that are left are read: none, one, some, just as many and one more; ties and
    infinities among them, said tokens, biases."""
    rng = np.random.default_rng(k)
    c = Case(41, typ, vocab, [9, 7], hist=60, few=vocab, bias=2, masks=16, mask_of=False, pad=pad)
    bits = np.zeros((16, -(-vocab // 32) * 32), bool)
    for row, n in enumerate([0, 1, 5, 31, 200, vocab // 33, vocab // 32, vocab // 32 + 2, vocab // 20, vocab // 64, 3, 3, 40, 40, 900, 900]):
        bits[row, rng.permutation(vocab)[:n]] = True
    bits[10, vocab - 1] = bits[11, 0] = True
    bits[12, :vocab] = rng.random(vocab) < 0.01
    said = c.r["history"][0, :20]
    bits[13, said[(said >= 0) & (said < vocab)]] = True
    c.r["allowed"] = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
    left = np.flatnonzero(bits[14, :vocab])
    c.logits[14, torch.from_numpy(left[:300]).cuda()] = 2.5
    c.logits[15, torch.from_numpy(np.flatnonzero(bits[15, :vocab])[:4]).cuda()] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0], device="cuda").to(c.logits.dtype)
    c.host = c.logits.float().cpu().numpy()
    check(ssd, c, k)


@pytest.mark.parametrize("k", [1, 5])
@pytest.mark.parametrize("typ,vocab,n", [("f16", 262144, 8), ("bf16", 66001, 320), ("f32", 9001, 16)])
def test_masks_that_leave_an_eighth(ssd, k, typ, vocab, n):
    """As many tokens as are taken as a list, some fewer and more; slices as large as lists can be."""
    rng = np.random.default_rng(n)
    c = Case(43, typ, vocab, None, n=n, hist=90, few=vocab, tokens=False, bias=2, masks=8)
    bits = np.zeros((8, -(-vocab // 32) * 32), bool)
    for i, step in enumerate((7, 8, 9)):
        bits[i, i:vocab:step] = True
    for i, share in enumerate((0.1, 0.124, 0.126, 0.3, 0.06)):
        bits[3 + i, :vocab] = rng.random(vocab) < share
    c.r["allowed"] = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
    check(ssd, c, k, want_adjust=False)


def test_infinities_and_nan(ssd):
    c = Case(2, "f32", 3333, [5], hist=40, few=20, masks=3)
    c.r["allowed_of"][:] = -1
    c.logits[0, 5], c.logits[0, 3000] = float("inf"), float("inf")
    c.logits[1, ::2] = float("nan")
    c.logits[2, 1:] = -float("inf")
    c.logits[3] = 3e38
    c.logits[4, 17] = -3e38
    c.host = c.logits.cpu().numpy()
    check(ssd, c, 6)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_rows_of_the_lowest_value(ssd, typ):
    """Masks that were made with the type's lowest value instead of -inf: tokens like any other."""
    c = Case(5, typ, 5003, [4], hist=0, tokens=False)
    c.logits[:] = torch.finfo(TYPES[typ]).min
    c.logits[1, 4000] = -1.0
    c.logits[2, ::2] = -float("inf")
    c.logits[3, 1:] = -float("inf")
    c.host = c.logits.float().cpu().numpy()
    for k in (1, 3):
        check(ssd, c, k, want_adjust=False)


def test_more_rows_than_a_grid_axis_has(ssd):
    n, vocab = 70001, 37
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(n, vocab, device="cuda", generator=g)
    bias = torch.randn(2, vocab, device="cuda", generator=g)
    rules = ssd.LogitRules(vocab, n, bias=bias, bias_of=(torch.arange(n, device="cuda") % 2).int())
    tokens, logprob, total, out = torch.empty(n, 2, dtype=torch.int32, device="cuda"), torch.empty(n, 2, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(x)
    ssd.ssd_logits_choose(rules, x, tokens, logprob, total, stream())
    ssd.ssd_logits_adjust(rules, x, out, stream())
    torch.cuda.synchronize()
    want = x + bias[torch.arange(n, device="cuda") % 2]
    assert torch.equal(out, want)
    top = torch.sort(want, dim=-1, descending=True, stable=True)
    assert torch.equal(tokens, top[1][:, :2].int())
    sums = torch.logsumexp(want.double(), -1)
    # (logits under 16, sums of 37 weights: 64 roundings of values under 16)
    assert float((total.double() - sums).abs().max()) < 64 * 16 * 2.0**-24
    assert float((logprob.double() - (top[0][:, :2].double() - sums[:, None])).abs().max()) < 64 * 16 * 2.0**-24


def test_an_ascending_row(ssd):
    """The best are all of one thread's chunk, and the last thread's best is the row's worst."""
    c = Case(3, "f32", 30000, [3], tokens=False)
    c.logits[0] = torch.arange(30000, device="cuda").float()
    c.logits[1] = -torch.arange(30000, device="cuda").float()
    c.logits[2] = (torch.arange(30000, device="cuda") // 8 % 512 == 77).float() * 10 + torch.arange(30000, device="cuda").float() * 1e-4
    c.host = c.logits.cpu().numpy()
    check(ssd, c, 16, want_adjust=False)


def test_rows_before_an_aligned_address(ssd):
    """Logits that start anywhere."""
    c = Case(4, "bf16", 1003, [6], hist=50, few=100, masks=3, bias=2)
    for off in (1, 5, 7):
        flat = torch.zeros(6 * 1009 + off, dtype=torch.bfloat16, device="cuda")
        view = flat[off:].view(6, 1009)[:, :1003]
        view.copy_(c.logits)
        d = Case(4, "bf16", 1003, [6], hist=50, few=100, masks=3, bias=2)
        d.logits = view
        check(ssd, d, 3)


def test_adjust_in_place(ssd):
    c = Case(6, "f16", 9001, [9, 8], hist=100, few=200, masks=4, bias=2)
    out = torch.empty_like(c.logits)
    ssd.ssd_logits_adjust(c.rules(ssd), c.logits, out, stream())
    keep = c.logits.clone()
    ssd.ssd_logits_adjust(c.rules(ssd), keep, keep, stream())
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), keep.view(torch.int16))


def test_a_replay_reads_lengths_and_starts_anew(ssd):
    c, d = (Case(s, "f32", 12000, [7, 9, 4], hist=200, few=100, masks=4) for s in (7, 8))
    rules, bufs = c.rules(ssd), (torch.empty(20, 4, dtype=torch.int32, device="cuda"), torch.empty(20, 4, device="cuda"), torch.empty(20, device="cuda"))
    logits = c.logits.contiguous().clone()
    ssd.ssd_logits_choose(rules, logits, *bufs, stream())  # (sets the kernels up)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ssd.ssd_logits_choose(rules, logits, *bufs, torch.cuda.current_stream().cuda_stream)
        ssd.ssd_logits_adjust(rules, logits, logits, torch.cuda.current_stream().cuda_stream)
    # the other case's contents: other lengths, other rows to the requests
    d.start = np.array([0, 4, 13, 20], np.int32)
    d.r["masks"] = tree_masks(np.random.default_rng(9), [4, 9, 7], 1)
    for t, name in zip(rules.keep, ("row_start", "history", "history_len", "prompt_len", "tokens", "masks", "repetition", "presence", "frequency", "bias", "bias_of", "allowed",
                                    "allowed_of")):
        if t is not None:
            t.copy_(gpu(d.start if name == "row_start" else d.r[name]))
    logits.copy_(d.logits)
    g.replay()
    torch.cuda.synchronize()
    for x, y in zip(bufs, check(ssd, d, 4)):
        assert torch.equal(x, y)
    assert torch.equal(torch.nan_to_num(logits), torch.nan_to_num(torch.from_numpy(d.expected()).cuda()))


def test_rows_beyond_32_bits(ssd):
    far = (1 << 31) + 5
    big = torch.zeros(2 * far + 3001, dtype=torch.float16, device="cuda")
    c, d = (Case(31, "f16", 3001, [2, 1], hist=40, few=100, masks=4, bias=2) for _ in range(2))
    d.logits = torch.as_strided(big, (3, 3001), (far, 1))
    d.logits.copy_(c.logits)
    for x, y in zip(check(ssd, c, 5), check(ssd, d, 5)):
        assert torch.equal(x, y)
    out = torch.empty_like(c.logits)
    ssd.ssd_logits_adjust(c.rules(ssd), c.logits, out, stream())
    ssd.ssd_logits_adjust(d.rules(ssd), d.logits, d.logits, stream())
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), d.logits.contiguous().view(torch.int16))


def test_two_streams_at_once(ssd):
    cs = [Case(20 + i, "bf16", 20000, [9] * 12, hist=100, few=100, masks=4) for i in range(2)]
    rules = [c.rules(ssd) for c in cs]
    outs = [[(torch.empty(c.n, 8, dtype=torch.int32, device="cuda"), torch.empty(c.n, 8, device="cuda"), torch.empty(c.n, device="cuda")) for _ in range(6)] for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for i in range(6):
        for c, r, o, s in zip(cs, rules, outs, streams):
            ssd.ssd_logits_choose(r, c.logits, *o[i], s.cuda_stream)
    torch.cuda.synchronize()
    for c, o in zip(cs, outs):
        want = check(ssd, c, 8, want_adjust=False)
        for got in o:
            assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_the_binding_refuses(ssd):
    c = Case(1, "f32", 64, [2, 2], hist=5)
    ok = c.rules(ssd)
    tok, lp = torch.empty(4, 2, dtype=torch.int32, device="cuda"), torch.empty(4, 2, device="cuda")
    for bad in (dict(logits=c.logits.half().double()), dict(logits=c.logits[:3]), dict(logits=c.logits.t().contiguous().t()), dict(tokens=tok[:3]), dict(tokens=tok.long()),
                dict(logprob=lp.half()), dict(logits=c.logits.cpu()), dict(total=torch.empty(3, device="cuda"))):
        a = {"logits": c.logits, "tokens": tok, "logprob": lp, "total": None, **bad}
        with pytest.raises(ssd.SSDError):
            ssd.ssd_logits_choose(ok, a["logits"], a["tokens"], a["logprob"], a["total"])
    for bad in (dict(history=None), dict(history_len=None), dict(presence=torch.ones(3, device="cuda")), dict(bias=torch.ones(1, 63, device="cuda")),
                dict(allowed=torch.ones(1, 1, dtype=torch.int32, device="cuda")), dict(bias_of=torch.zeros(2, dtype=torch.int32, device="cuda")),
                dict(masks=torch.zeros(4, dtype=torch.int64, device="cuda")), dict(tokens=torch.zeros(4, dtype=torch.int64, device="cuda")), dict(repetition=torch.ones(2))):
        with pytest.raises(ssd.SSDError):
            ssd.LogitRules(64, 4, **{**dict(row_start=gpu(c.start), max_rows=2, **{k: gpu(v) for k, v in c.r.items()}), **bad})
