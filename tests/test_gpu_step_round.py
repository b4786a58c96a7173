"""The operators as a program uses them together: a round of greedy decoding over drafted trees, for a small decoder whose layers
normalise their heads, have positions on three axes and a mixture of experts, with penalised and masked choices.

Everything between the operators (projections, norms of rows) is plain PyTorch in the test.  The first round is checked step by step
against numpy in 64 bits; then rounds run in a captured graph, with the same bits as eager ones, until texts have grown by several commits.
"""
import numpy as np
import pytest

import step_reference as step
import tree_reference as tree

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

L, D, H, G, HD, F, E, K, V, PAGE, PAGES = 2, 128, 4, 2, 64, 72, 8, 2, 301, 16, 64
B, NODES, HIST = 3, [5, 1, 7], 64
T, EPS = torch.float16, 1e-5
SECTIONS = [12, 10, 10]


@pytest.fixture(scope="module")
def ssd():
    import paper_2309_08168_gb300 as m
    return m


def f64(t):
    return t.double().cpu().numpy()


class Round:
    def __init__(self, ssd):
        g = torch.Generator().manual_seed(4)
        self.ssd, n = ssd, sum(NODES)

        def normal(*s, std):
            return (std * torch.randn(*s, generator=g)).to(T).cuda()
        self.w = [dict(qkv=normal((H + 2 * G) * HD, D, std=D**-0.5), o=normal(D, H * HD, std=(H * HD) ** -0.5), router=normal(E, D, std=D**-0.5),
                       experts=ssd.MoeWeights(normal(E, F, D, std=D**-0.5), normal(E, F, D, std=D**-0.5), normal(E, D, F, std=F**-0.5)),
                       norm=ssd.HeadNorm((1 + 0.2 * torch.randn(HD, generator=g)).cuda(), (1 + 0.2 * torch.randn(HD, generator=g)).cuda(), EPS)) for _ in range(L)]
        self.embed, self.head = normal(V, D, std=1.0), normal(V, D, std=2 * D**-0.5)
        self.kv = ssd.PagedKV(*(torch.zeros(L, PAGES, G, PAGE, HD, dtype=T, device="cuda") for _ in range(2)))
        self.rope = ssd.ssd_rope_init(HD, 1e4)
        self.axes = ssd.ssd_rope_axes_init(self.rope, ssd.SSD_AXES_SECTIONS, SECTIONS)

        def ints(v):
            return torch.tensor(v, dtype=torch.int32, device="cuda")
        self.lens, self.held = ints([0, 0, 0]), ints([0, 0, 0])
        self.start = ints([0, *np.cumsum(NODES)])
        self.table, self.ring = torch.full((B, 12), -1, dtype=torch.int32, device="cuda"), torch.arange(PAGES, dtype=torch.int32, device="cuda")
        self.ends = torch.tensor([0, PAGES], device="cuda")
        self.parents = ints([-1, 0, 0, 1, 3, -1, -1, 0, 1, 0, 3, 4, 2])
        self.batch = ssd.TreeBatch(self.start, self.lens, self.table, n, max(NODES))
        self.held2, self.ends2, self.lens2 = ints([0] * B), torch.zeros_like(self.ends), ints([0] * B)
        self.slots, self.positions, self.status = ints([0] * n), ints([0] * n), ints([0])
        self.masks = torch.zeros(n, 1, dtype=torch.int64, device="cuda")
        self.attention_ws = torch.empty(ssd.ssd_tree_attention_workspace(self.kv), dtype=torch.uint8, device="cuda")
        self.moe_ws = torch.empty(ssd.ssd_moe_workspace(self.w[0]["experts"], n, K), dtype=torch.uint8, device="cuda")
        self.tokens = torch.randint(0, V, (n,), generator=g).int().cuda()
        self.history = torch.randint(0, V, (B, HIST), generator=g).int().cuda()
        self.history_len, self.prompt_len = ints([9, 4, 0]), ints([6, 4, 0])
        allowed = torch.randint(-2**31, 2**31, (2, -(-V // 32)), generator=g).int()
        allowed[1] = -1
        self.allowed, self.allowed_of = allowed.cuda(), ints([0, 1] * (n // 2) + [1] * (n % 2))
        self.bias = (2 * torch.randn(1, V, generator=g)).cuda()
        self.rules = ssd.LogitRules(V, n, row_start=self.start, max_rows=max(NODES), history=self.history, history_len=self.history_len, prompt_len=self.prompt_len,
                                    tokens=self.tokens, masks=self.masks, repetition=torch.full((B,), 1.3, device="cuda"), presence=torch.full((B,), 0.25, device="cuda"),
                                    frequency=torch.full((B,), 0.5, device="cuda"), bias=self.bias, allowed=self.allowed, allowed_of=self.allowed_of)
        self.best, self.logprob, self.total = (torch.zeros(n, 3, dtype=d, device="cuda") if i < 2 else torch.zeros(n, device="cuda") for i, d in
                                               enumerate((torch.int32, torch.float32, None)))
        self.ids, self.weights = torch.zeros(n, K, dtype=torch.int32, device="cuda"), torch.zeros(n, K, device="cuda")
        self.q, self.att = (torch.zeros(n, H, HD, dtype=T, device="cuda") for _ in range(2))
        self.out = torch.zeros(n, D, dtype=T, device="cuda")
        self.accepted, self.next = ints([0] * B), ints([0] * B)
        self.path, self.emitted = ints([0] * n), ints([0] * n)
        self.seen = []  # what the first round is checked by

    def run(self, watch=False):
        s, ssd, n = torch.cuda.current_stream().cuda_stream, self.ssd, self.tokens.numel()
        ssd.ssd_tree_plan(self.batch, PAGE, PAGES, self.parents, self.held, self.held2, self.ring, self.ends, self.ends2, self.slots, self.positions, self.masks, self.status, s)
        # text has its position on every axis (an image's pieces would not)
        positions = torch.stack([self.positions, self.positions // 2, self.positions % 3])
        x = self.embed[self.tokens.long()]
        for i, w in enumerate(self.w):
            y = x / x.float().square().mean(-1, keepdim=True).sqrt().to(T)
            qkv = y @ w["qkv"].t()
            q, k, v = (t.unflatten(1, (-1, HD)) for t in qkv.split([H * HD, G * HD, G * HD], 1))
            ssd.ssd_norm_rope_kv(self.kv, i, self.rope, q, k, v, positions, self.slots, self.q, axes=self.axes, norm=w["norm"], cuda_stream=s)
            ssd.ssd_tree_attention(self.batch, self.kv, i, self.q, self.masks, HD**-0.5, self.att, self.attention_ws, self.status, s)
            x = x + self.att.flatten(1) @ w["o"].t()
            y = x / x.float().square().mean(-1, keepdim=True).sqrt().to(T)
            ssd.ssd_moe_route(y, w["router"], self.ids, self.weights, cuda_stream=s)
            ssd.ssd_moe_mlp(w["experts"], y, self.ids, self.weights, self.out, self.moe_ws, residual=x, status=self.status, cuda_stream=s)
            if watch:
                torch.cuda.synchronize()
                self.seen.append({a: b.clone() for a, b in dict(q=q, k=k, v=v, positions=positions, q_out=self.q, att=self.att, y=y, x=x, ids=self.ids, weights=self.weights, out=self.out).items()})
            x = self.out.clone()
        logits = x @ self.head.t()
        ssd.ssd_logits_choose(self.rules, logits, self.best, self.logprob, self.total, s)
        target = self.best[:, 0].contiguous()
        ssd.ssd_tree_commit(self.batch, self.kv, self.parents, self.tokens, target, self.accepted, self.next, self.lens2, self.path, self.emitted, s)
        if watch:
            torch.cuda.synchronize()
            self.logits, self.target = logits.clone(), target.clone()
        # the next round starts from the committed texts: their tokens join the history, the next token is the root, and drafts are the
        # second and third best of the root's row and so on (what they are does not matter here)
        at = torch.arange(HIST, device="cuda")
        first = self.history_len
        for b in range(B):
            r0 = int(np.cumsum([0] + NODES)[b])
            j = at - first[b]
            row = (self.path[r0:r0 + NODES[b]] + r0).long()[j.clamp(0, NODES[b] - 1)]
            self.history[b] = torch.where((j >= 0) & (j <= self.accepted[b]), self.tokens[row], self.history[b])
        self.history_len += self.accepted + 1
        self.lens.copy_(self.lens2)
        self.held.copy_(self.held2)
        self.ends.copy_(self.ends2)
        drafts = self.best.flatten()[: n].clamp(min=0)
        for b in range(B):
            r0 = int(np.cumsum([0] + NODES)[b])
            self.tokens[r0:r0 + NODES[b]] = drafts[r0:r0 + NODES[b]]
            self.tokens[r0:r0 + 1] = self.next[b:b + 1]

    def state(self):
        return [t.clone() for t in (self.kv.k, self.kv.v, self.lens, self.table, self.history, self.history_len, self.tokens, self.best, self.logprob, self.emitted, self.status)]


def test_a_round_step_by_step(ssd):
    r = Round(ssd)
    tokens, history, lens = r.tokens.cpu().numpy().copy(), r.history.cpu().numpy().copy(), r.history_len.cpu().numpy().copy()
    r.run(watch=True)
    start, n = [0, *np.cumsum(NODES)], sum(NODES)
    masks = r.masks.cpu().numpy()
    rates, axis = tree.frequencies(HD, 1e4), step.axis_of_pair(HD // 2, 3, SECTIONS, False)
    for i, s in enumerate(r.seen):
        gains = [t.cpu().numpy() for t in r.w[i]["norm"].keep]
        for row in range(n):
            pos = s["positions"][:, row].tolist()
            for name, got, gain in (("q", s["q_out"][row], gains[0]), ("k", r_cache(r.slots[row], s, r, i), gains[1])):
                if got is None:
                    continue
                want = step.turned(f64(s[name][row]), gain, EPS, pos, axis, rates, HD, False)
                # a rounding to fp16 and 20 of fp32 in a pair's parts
                assert np.abs(f64(got) - want).max() <= 2.0**-11 * np.abs(want).max() + 40 * 2.0**-24 * np.abs(want).max() * 2
        # attention over what the cache held then: one tree each, no prefix
        want = np.zeros((n, H, HD))
        for b in range(B):
            rows = range(start[b], start[b + 1])
            kk = np.stack([step.turned(f64(s["k"][x]), gains[1], EPS, s["positions"][:, x].tolist(), axis, rates, HD, False) for x in rows])
            vv = np.stack([f64(s["v"][x]) for x in rows])
            for x in rows:
                seen = [j for j in range(len(kk)) if (int(masks[x, 0]) >> j) & 1]
                for h in range(H):
                    g = h * G // H
                    z = kk[seen, g] @ f64(s["q_out"][x, h]) * HD**-0.5
                    w = np.exp(z - z.max())
                    want[x, h] = w @ vv[seen, g] / w.sum()
        # keys are rounded to fp16 in the cache: a score is off by at most 2^-11 of its absolute terms (under 8 here), a weight by that
        assert np.abs(f64(s["att"]) - want).max() <= (2 * 8 * 2.0**-11 + 2.0**-11 + 1e-4) * np.abs(f64(s["v"])).max()
        ids, p = step.routed(f64(s["y"]), f64(r.w[i]["router"]), K, None, False, True, 1.0)
        assert np.array_equal(s["ids"].cpu().numpy(), ids)
        np.testing.assert_allclose(f64(s["weights"]), p, rtol=16 * 2.0**-24)
        gate, up, down = (f64(t) for t in r.w[i]["experts"].keep)
        want, err = step.mlp(f64(s["y"]), ids, f64(s["weights"]), gate, up, down, f64(s["x"]), 2.0**-11)
        assert (np.abs(f64(s["out"]) - want) <= err + 2.0**-11 * (np.abs(want) + err) + 2.0**-25).all()
    rules = dict(history=history, history_len=lens, prompt_len=r.prompt_len.cpu().numpy(), tokens=tokens, masks=masks, repetition=np.full(B, 1.3, np.float32),
                 presence=np.full(B, 0.25, np.float32), frequency=np.full(B, 0.5, np.float32), bias=r.bias.cpu().numpy(), allowed=r.allowed.cpu().numpy(),
                 allowed_of=r.allowed_of.cpu().numpy())
    logits, best = r.logits.float().cpu().numpy(), r.best.cpu().numpy()
    for b in range(B):
        for row in range(start[b], start[b + 1]):
            want = step.adjusted(logits[row], V, b, row, row - start[b], start[b], NODES[b], rules)
            assert best[row].tolist() == step.chosen(want, 3)[0]
    acc, nxt, new, path, emitted, _ = tree.commit(start, np.zeros(B, np.int32), r.table.cpu().numpy(), PAGE, r.parents.cpu().numpy(), tokens, r.target.cpu().numpy(), n)
    assert np.array_equal(r.accepted.cpu().numpy(), acc) and np.array_equal(r.next.cpu().numpy(), nxt) and np.array_equal(r.lens.cpu().numpy(), new)
    assert r.status.item() == 0


def r_cache(slot, s, r, layer):
    """A key as the cache holds it, where the commit has not moved anything over it (its row may have been; then None)."""
    return None if layer < L - 1 or r.accepted.max() > 0 else r.kv.k[layer, int(slot) // PAGE, :, int(slot) % PAGE]


def test_rounds_in_a_graph(ssd):
    """Texts that grow by commits: the captured round has the bits of the eager one, round after round."""
    a, b = Round(ssd), Round(ssd)
    side = torch.cuda.Stream()
    a.run()
    b.run()  # (sets the kernels up)
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        b.run()
    for i in range(7):
        a.run()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(torch.nan_to_num(x.float()), torch.nan_to_num(y.float())), i
    assert a.status.item() == 0 and (a.lens.cpu().numpy() >= 8).all()
