"""The operators of a decoding step around the tree operators, as they are measured.

Four kinds of case:

  heads   ssd_norm_rope_kv: queries and keys normalised head by head and turned to positions on one or several axes, keys and values
          written to their cache rows
  adjust  ssd_logits_adjust: penalties for tokens that were said before, biases and masks of allowed tokens on logits
  choose  ssd_logits_choose: the same, and the k best tokens of every row with their log probabilities
  moe     ssd_moe_route and ssd_moe_mlp: a mixture-of-experts layer for a few rows

Lengths and row counts of a batch follow from the case alone (the work of a case
has to be known without its inputs); everything else is made from the seed.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SAID = (1.3, 0.4, 0.2)  # repetition, presence and frequency penalties, about


def listed():
    return [
        # one decoding step of a single request with grouped heads at 70B widths: latency only
        dict(name="heads_step", kind="heads", type="bf16", heads=64, kv_heads=8, hd=128, n=1, rot=128, pairs="half", axes=1, norm="both"),
        # trees of a batch behind images: three axes by sections, normalised heads
        dict(name="heads_tree", kind="heads", type="f16", heads=32, kv_heads=8, hd=128, n=403, rot=128, pairs="half", axes=3, norm="both"),
        # a long prompt with images, fp32 rows, part of every head rotated, axes in turns
        dict(name="heads_prompt", kind="heads", type="f32", heads=32, kv_heads=32, hd=128, n=4095, rot=64, pairs="neighbours", axes=2, norm="both"),
        # the choice of a verification at 7B's vocabulary, nothing to adjust: 9 rows
        dict(name="choose_small", kind="choose", type="f32", vocab=32000, n=1, rows=9, tree=True, hist=0, k=1, bias=0, masks=0),
        # drafting: eight children for every node of a batch's trees, said tokens penalised, an odd vocabulary
        dict(name="choose_tree", kind="choose", type="bf16", vocab=50257, n=8, rows=33, tree=True, hist=900, k=8, bias=2, masks=0),
        # single tokens of a large batch with a grammar each, a large vocabulary, long histories
        dict(name="choose_batch", kind="choose", type="f16", vocab=128256, n=512, rows=1, tree=False, hist=4000, k=1, bias=3, masks=64),
        # logits of a few requests made ready for a sampler of the user's
        dict(name="adjust_step", kind="adjust", type="f32", vocab=32000, n=4, rows=1, tree=False, hist=300, k=0, bias=1, masks=3),
        # and of a batch's trees
        dict(name="adjust_tree", kind="adjust", type="bf16", vocab=151936, n=24, rows=17, tree=True, hist=2500, k=0, bias=0, masks=40),
        # one token, two of eight experts at 7B widths: the weights are all there is
        dict(name="moe_step", kind="moe", type="bf16", n=1, d=4096, f=11008, experts=8, k=2, score="softmax"),
        # a chain of drafts verified, many small experts
        dict(name="moe_verify", kind="moe", type="bf16", n=9, d=2048, f=768, experts=128, k=8, score="softmax"),
        # a tree of 33 nodes, scores by sigmoid with a bias, odd sizes
        dict(name="moe_tree", kind="moe", type="f16", n=33, d=4104, f=1416, experts=64, k=6, score="sigmoid"),
        # the trees of several requests at 13B widths
        dict(name="moe_batch", kind="moe", type="bf16", n=64, d=5120, f=13824, experts=16, k=2, score="softmax"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["heads", "heads", "adjust", "choose", "choose", "choose", "moe", "moe", "moe"])
    typ = rng.choice(["f32", "f16", "bf16"])
    if kind == "heads":
        hd = rng.choice([64, 128, 128])
        kv = _log(rng, 1, 40)
        group = rng.choice([1, 1, 2, 4, 5, 8])
        if kv * group > 64:
            kv = 64 // group
        n = _log(rng, 1, min(16000, 35_000_000 // (kv * (group + 2) * hd)))
        return dict(kind=kind, type=typ, heads=kv * group, kv_heads=kv, hd=hd, n=n, rot=rng.choice([hd, hd, hd // 2, hd // 4, 48]),
                    pairs=rng.choice(["half", "neighbours"]), axes=rng.choice([1, 2, 3, 3, 4]), norm=rng.choice(["both", "both", "q", "k", "none"]))
    if kind == "moe":
        while True:
            d, f, experts = 8 * _log(rng, 16, 1024), 8 * _log(rng, 2, 1800), _log(rng, 1, 256)
            if 1e5 <= d * f * experts <= 1.1e9:
                break
        return dict(kind=kind, type=rng.choice(["f16", "bf16"]), n=_log(rng, 1, 64), d=d, f=f, experts=experts, k=rng.randint(1, min(8, experts)),
                    score=rng.choice(["softmax", "softmax", "sigmoid"]))
    tree = rng.random() < 0.5
    vocab = _log(rng, 500, 260000)
    while True:
        n, rows = _log(rng, 1, 512), _log(rng, 1, 128) if tree else 1
        if n * rows * vocab <= 6.5e7:
            break
    return dict(kind=kind, type=typ, vocab=vocab, n=n, rows=rows, tree=tree, hist=rng.choice([0, _log(rng, 1, 8000), _log(rng, 1, 8000)]),
                k=0 if kind == "adjust" else rng.choice([1, 1, _log(rng, 2, 16)]), bias=rng.choice([0, 0, 1, 3]), masks=rng.choice([0, 0, _log(rng, 1, 64)]))


# -- sizes and inputs -----------------------------------------------------------

def _sizes(c):
    """(row counts, lengths of what was said) of the requests; the first is as long as they get."""
    rng = random.Random(1000 * c["n"] + c["rows"])
    rows = [c["rows"]] + [rng.randint((c["rows"] + 1) // 2, c["rows"]) for _ in range(c["n"] - 1)]
    hist = [c["hist"]] + [rng.randint(0, c["hist"]) for _ in range(c["n"] - 1)]
    return rows, hist


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"case": case, **{"heads": _prepare_heads, "moe": _prepare_moe}.get(case["kind"], _prepare_logits)(case, g)}


def _axis_of_pair(c):
    """Which axis turns each pair: sections of equal size (the first takes what is left), or in turns while an axis has pairs left."""
    half, axes = c["rot"] // 2, c["axes"]
    pairs = [half - (axes - 1) * (half // axes)] + [half // axes] * (axes - 1)
    if c["pairs"] == "half":
        return pairs, [a for a in range(axes) for _ in range(pairs[a])]
    return pairs, [i % axes if i // axes < pairs[i % axes] else 0 for i in range(half)]


def _prepare_heads(c, g):
    n, t = c["n"], _TYPES[c["type"]]
    width = [c["heads"] * c["hd"], c["kv_heads"] * c["hd"], c["kv_heads"] * c["hd"]]
    packed = (1.7 * torch.randn(n, sum(width), device="cuda", generator=g)).to(t)  # the projections' output, q then k then v
    n_pages = -(-n * 5 // 4 // 16) + 1
    cache = [torch.empty(1, n_pages, c["kv_heads"], 16, c["hd"], dtype=torch.float16 if c["type"] == "f32" else t, device="cuda").normal_(generator=g) for _ in range(2)]
    slots = torch.randperm(n_pages * 16, generator=g, device="cuda")[:n].int()
    if n > 1:
        slots[n // 2] = -1  # a row that has no place in the cache
    gains = [1.0 + 0.2 * torch.randn(c["hd"], device="cuda", generator=g) for _ in range(2)]
    s = {x: y.unflatten(1, (-1, c["hd"])) for x, y in zip("qkv", packed.split(width, 1))}
    s.update(cache=cache, slots=slots, positions=torch.randint(0, 40000, (c["axes"], n), generator=g, device="cuda").int(),
             gain={"q": gains[0] if c["norm"] in ("both", "q") else None, "k": gains[1] if c["norm"] in ("both", "k") else None},
             out=torch.empty(n, c["heads"], c["hd"], dtype=t, device="cuda"))
    if own:
        import paper_2309_08168_gb300 as ssd
        s["kv"] = ssd.PagedKV(*cache)
        s["rope"] = ssd.ssd_rope_init(c["rot"], theta=1e6, interleaved=c["pairs"] == "neighbours")
        s["axes"] = ssd.ssd_rope_axes_init(s["rope"], ssd.SSD_AXES_SECTIONS if c["pairs"] == "half" else ssd.SSD_AXES_IN_TURNS, _axis_of_pair(c)[0])
        s["norm"] = ssd.HeadNorm(s["gain"]["q"], s["gain"]["k"], 1e-6)
    return s


def _nodes(start, n):
    """(index within its request, request) of rows 0 .. n-1."""
    r = torch.arange(n, device=start.device)
    b = torch.searchsorted(start[1:].contiguous(), r.int(), right=True)
    return r - start.long()[b], b


def _reach(c, start, n, g):
    """[row][j]: whether node j is the row's node or above it in a random tree, parents in [i / 4, i)."""
    node, b = _nodes(start, n)
    lo = node // 4
    p = torch.minimum(lo + (torch.rand(n, device="cuda", generator=g) * (node - lo)).long(), node - 1)
    m = torch.eye(c["rows"], device="cuda").repeat(c["n"], 1, 1)
    m[b[node > 0], node[node > 0], p[node > 0]] = 1.0
    for _ in range(max(1, (c["rows"] - 1).bit_length())):  # (paths of twice the length each time)
        m = ((m @ m) > 0).float()
    return m[b, node] > 0


def _prepare_logits(c, g):
    rows, hist = _sizes(c)
    start = _ints([0] + torch.tensor(rows).cumsum(0).tolist())
    n, words = sum(rows), -(-c["vocab"] // 32)
    s = {"start": start, "n_rows": n, "logits": (3.0 * torch.randn(n, c["vocab"], device="cuda", generator=g)).to(_TYPES[c["type"]])}
    few = min(c["vocab"], 4000)  # texts use few of the tokens again and again
    s["tokens"] = (torch.rand(n, device="cuda", generator=g) ** 2 * few).int()
    s["masks"] = None
    if c["tree"]:
        w = -(-c["rows"] // 64)
        bits = torch.zeros(n, 64 * w, dtype=torch.int64, device="cuda")
        bits[:, :c["rows"]] = _reach(c, start, n, g).long()
        s["masks"] = (bits.view(n, w, 64) << torch.arange(64, device="cuda")).sum(-1)
    s["history"] = None
    if c["hist"]:
        s["history"] = (torch.rand(c["n"], c["hist"], device="cuda", generator=g) ** 2 * few).int()
        s["history_len"], s["prompt_len"] = _ints(hist), _ints([x // 2 for x in hist])
        s["said"] = [x * (0.5 + torch.rand(c["n"], device="cuda", generator=g)) for x in _SAID]
    s["bias"] = s["allowed"] = None
    if c["bias"]:
        bias = 4.0 * torch.randn(c["bias"], c["vocab"], device="cuda", generator=g)
        s["bias"] = torch.where(torch.rand(c["bias"], c["vocab"], device="cuda", generator=g) < 0.001, bias, 0.0)
        s["bias_of"] = torch.randint(-1, c["bias"], (c["n"],), generator=g, device="cuda").int()
    if c["masks"]:
        share = torch.rand(c["masks"], 1, device="cuda", generator=g) ** 4  # some grammars allow a few tokens, some most of them
        ok = torch.zeros(c["masks"], 32 * words, dtype=torch.bool, device="cuda")
        ok[:, :c["vocab"]] = torch.rand(c["masks"], c["vocab"], device="cuda", generator=g) < share
        ok[0, 1:] = False  # (the text has to end)
        s["allowed"] = (ok.view(c["masks"], words, 32).long() << torch.arange(32, device="cuda")).sum(-1).int()
        s["allowed_of"] = torch.randint(-1, c["masks"], (n,), generator=g, device="cuda").int()
    if c["kind"] == "adjust":
        s["out"] = torch.empty_like(s["logits"])
    else:
        s["best"] = torch.empty(n, c["k"], dtype=torch.int32, device="cuda")
        s["logprob"], s["total"] = torch.empty(n, c["k"], device="cuda"), torch.empty(n, device="cuda")
    if own:
        import paper_2309_08168_gb300 as ssd
        said = s["said"] if c["hist"] else (None, None, None)
        s["rules"] = ssd.LogitRules(c["vocab"], row_start=start, n_rows=n, max_rows=c["rows"], history=s["history"], history_len=s.get("history_len"),
                                    prompt_len=s.get("prompt_len"), tokens=s["tokens"] if c["hist"] else None, masks=s["masks"] if c["hist"] else None,
                                    repetition=said[0], presence=said[1], frequency=said[2], bias=s["bias"], bias_of=s.get("bias_of"),
                                    allowed=s["allowed"], allowed_of=s.get("allowed_of"))
    return s


def _prepare_moe(c, g):
    t, d, f, e = _TYPES[c["type"]], c["d"], c["f"], c["experts"]

    def normal(*shape, std=1.0):
        return torch.empty(*shape, dtype=t, device="cuda").normal_(0.0, std, generator=g)
    s = {"x": normal(c["n"], d), "router": normal(e, d, std=d ** -0.5), "gate": normal(e, f, d, std=d ** -0.5), "up": normal(e, f, d, std=d ** -0.5),
         "down": normal(e, d, f, std=f ** -0.5), "residual": normal(c["n"], d), "favour": None}
    if c["score"] == "sigmoid":
        s["favour"] = 0.1 * torch.randn(e, device="cuda", generator=g)
    s["ids"] = torch.empty(c["n"], c["k"], dtype=torch.int32, device="cuda")
    s["weights"] = torch.empty(c["n"], c["k"], device="cuda")
    s["out"] = torch.empty_like(s["x"])
    if own:
        import paper_2309_08168_gb300 as ssd
        s["experts"] = ssd.MoeWeights(s["gate"], s["up"], s["down"])
        s["workspace"] = torch.empty(ssd.ssd_moe_workspace(s["experts"], c["n"], c["k"]), dtype=torch.uint8, device="cuda")
    return s


# -- one pass ---------------------------------------------------------------------

def run(state):
    return {"heads": _run_heads, "adjust": _run_adjust, "choose": _run_choose, "moe": _run_moe}[state["case"]["kind"]](state["case"], state)


def _run_heads(c, s):
    if own:
        import paper_2309_08168_gb300 as ssd
        ssd.ssd_norm_rope_kv(s["kv"], 0, s["rope"], s["q"], s["k"], s["v"], s["positions"], s["slots"], s["out"], axes=s["axes"], norm=s["norm"],
                             cuda_stream=torch.cuda.current_stream().cuda_stream)
        return [s["out"], *s["cache"]]
    f = 1e6 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda") / c["rot"])
    angle = s["positions"].double()[_axis_of_pair(c)[1]].t() * f
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def ready(name):
        x, r, h = s[name].float(), c["rot"], c["rot"] // 2
        if s["gain"][name] is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * s["gain"][name]
        if c["pairs"] == "half":
            a, b = x[..., :h], x[..., h:r]
            return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., r:]], -1)
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., r:]], -1)
    keys, values = s["cache"]
    has = s["slots"] >= 0
    page, at = s["slots"].long()[has] // 16, s["slots"].long()[has] % 16
    keys[0, page, :, at] = ready("k")[has].to(keys.dtype)
    values[0, page, :, at] = s["v"][has].to(values.dtype)
    return [ready("q").to(s["q"].dtype), keys, values]


def _adjusted(c, s):
    """The logits after penalties, biases and masks, in 32 bits."""
    x, v = s["logits"].float(), c["vocab"]
    node, b = _nodes(s["start"], s["n_rows"])
    if c["hist"]:
        at = torch.arange(c["hist"], device="cuda")[None]
        spoken = (at >= s["prompt_len"][:, None]) & (at < s["history_len"][:, None])
        prompt = at < s["prompt_len"][:, None]
        zero = torch.zeros(c["n"], v, dtype=torch.int32, device="cuda")
        count = zero.scatter_add(1, s["history"].long(), spoken.int())[b]
        seen = zero.scatter_add(1, s["history"].long(), prompt.int())[b]
        j = torch.arange(c["rows"], device="cuda").expand(s["n_rows"], -1)
        if s["masks"] is None:
            above = j <= node[:, None]
        else:
            above = (s["masks"].gather(1, j // 64) >> (j % 64)) & 1 == 1
        said = s["tokens"].long()[(s["start"].long()[b][:, None] + j).clamp(max=s["n_rows"] - 1)]
        count.scatter_add_(1, said, above.int())
        again, once, often = (p[b][:, None] for p in s["said"])
        x = torch.where((count > 0) | (seen > 0), torch.where(x > 0, x / again, x * again), x)
        x = x - often * count
        x = x - torch.where(count > 0, once, 0.0)
    if c["bias"]:
        x = x + torch.where(s["bias_of"][b][:, None] >= 0, s["bias"][s["bias_of"].long()[b].clamp(min=0)], 0.0)
    if c["masks"]:
        t = torch.arange(v, device="cuda")
        ok = (s["allowed"][s["allowed_of"].long().clamp(min=0)][:, t // 32] >> (t % 32)) & 1 == 1
        x = torch.where(ok | (s["allowed_of"][:, None] < 0), x, -math.inf)
    return x


def _run_adjust(c, s):
    if own:
        import paper_2309_08168_gb300 as ssd
        ssd.ssd_logits_adjust(s["rules"], s["logits"], s["out"], torch.cuda.current_stream().cuda_stream)
        return s["out"]
    return _adjusted(c, s).to(s["logits"].dtype)


def _run_choose(c, s):
    if own:
        import paper_2309_08168_gb300 as ssd
        ssd.ssd_logits_choose(s["rules"], s["logits"], s["best"], s["logprob"], s["total"], torch.cuda.current_stream().cuda_stream)
        return {"best": s["best"], "logprob": s["logprob"], "total": s["total"]}
    x = _adjusted(c, s)
    if c["k"] == 1:
        top = x.amax(-1, keepdim=True)
        best = (x == top).int().argmax(-1, keepdim=True)  # the lowest of those that tie
    else:
        top, best = torch.sort(x, dim=-1, descending=True, stable=True)
        top, best = top[:, :c["k"]], best[:, :c["k"]]
    none = top == -math.inf  # (a row whose mask leaves nothing has no best token and a sum of zero)
    m = torch.where(none[:, :1], 0.0, top[:, :1])
    total = torch.exp(x - m).sum(-1, keepdim=True).log()
    return {"best": torch.where(none, -1, best).int(), "logprob": torch.where(none, -math.inf, top - m - total), "total": (m + total)[:, 0]}


def _run_moe(c, s):
    if own:
        import paper_2309_08168_gb300 as ssd
        stream = torch.cuda.current_stream().cuda_stream
        ssd.ssd_moe_route(s["x"], s["router"], s["ids"], s["weights"], score=ssd.SSD_MOE_SOFTMAX if c["score"] == "softmax" else ssd.SSD_MOE_SIGMOID,
                          favour=s["favour"], renorm=True, cuda_stream=stream)
        ssd.ssd_moe_mlp(s["experts"], s["x"], s["ids"], s["weights"], s["out"], s["workspace"], residual=s["residual"], cuda_stream=stream)
        return {"ids": s["ids"], "weights": s["weights"], "out": s["out"]}
    # which experts come next to one another has to be right to the last bits: 64 of them
    logits = s["x"].double() @ s["router"].double().t()
    p = 1.0 / (1.0 + torch.exp(-logits)) if c["score"] == "sigmoid" else torch.exp(logits - logits.amax(-1, keepdim=True))
    if c["score"] == "softmax":
        p = p / p.sum(-1, keepdim=True)
    order = torch.sort(p if s["favour"] is None else p + s["favour"], dim=-1, descending=True, stable=True)[1][:, :c["k"]]
    w = p.gather(1, order)
    w = (w / w.sum(-1, keepdim=True)).float()
    x = s["x"].float()
    if c["n"] * c["k"] < c["experts"]:
        # few pairs of a row and an expert: their weights, pair by pair
        e = order.flatten()
        xe = x.repeat_interleave(c["k"], 0)[:, :, None]
        a, u = s["gate"][e].float() @ xe, s["up"][e].float() @ xe
        y = (s["down"][e].float() @ (a / (1.0 + torch.exp(-a)) * u)).view(c["n"], c["k"], -1)
        out = s["residual"].float() + (w[:, :, None] * y).sum(1)
    else:
        a, u = x @ s["gate"].float().transpose(1, 2), x @ s["up"].float().transpose(1, 2)
        y = (a / (1.0 + torch.exp(-a)) * u) @ s["down"].float().transpose(1, 2)  # [expert][row][d]
        share = torch.zeros(c["n"], c["experts"], device="cuda").scatter(1, order, w)
        out = s["residual"].float() + (share.t()[:, :, None] * y).sum(0)
    return {"ids": order.int(), "weights": w, "out": out.to(s["x"].dtype)}


# -- the work of one pass -----------------------------------------------------------

def work(case):
    c = case
    e = 4 if c["type"] == "f32" else 2
    if c["kind"] == "heads":
        row = c["hd"] * (e * (2 * c["heads"] + 2 * c["kv_heads"]) + 2 * 2 * c["kv_heads"])
        return {"bytes": float(c["n"] * (row + 4 + 4 * c["axes"])), "flops": float(c["n"] * (c["heads"] + c["kv_heads"]) * (3 * c["rot"] + 4 * c["hd"]))}
    if c["kind"] == "moe":
        met = c["experts"] * (1.0 - (1.0 - c["k"] / c["experts"]) ** c["n"])  # experts that some row goes to, about
        weights = 3.0 * met * c["d"] * c["f"] + c["experts"] * c["d"]
        return {"bytes": e * (weights + 3.0 * c["n"] * c["d"]) + 8.0 * c["n"] * c["k"],
                "flops": c["n"] * (6.0 * c["k"] * c["d"] * c["f"] + 2.0 * c["experts"] * c["d"])}
    rows, hist = _sizes(c)
    n = sum(rows)
    size = n * c["vocab"] * e * (2 if c["kind"] == "adjust" else 1) + 4.0 * sum(hist) + c["bias"] * c["vocab"] * 4.0 + min(c["masks"], n) * c["vocab"] / 8
    return {"bytes": float(size + n * (4 + 8 * c["k"])), "flops": 2.0 * n * c["vocab"]}


# -- the same in 64 bits --------------------------------------------------------------

def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "heads":
        place = torch.tensor(_axis_of_pair(c)[1], device="cuda")
        rate = torch.tensor([1e6 ** (-2 * i / c["rot"]) for i in range(c["rot"] // 2)], dtype=torch.float64, device="cuda")
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[place].t() * rate)[:, None]
        out = []
        for name in "qk":
            x, h = s[name].double(), c["rot"] // 2
            if s["gain"][name] is not None:
                x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / c["hd"] + 1e-6) * s["gain"][name].double()
            lo, hi = (slice(0, h), slice(h, 2 * h)) if c["pairs"] == "half" else (slice(0, 2 * h, 2), slice(1, 2 * h, 2))
            y = torch.complex(x[..., lo].contiguous(), x[..., hi].contiguous()) * z
            x = x.clone()
            x[..., lo], x[..., hi] = y.real, y.imag
            out.append(x)
        keys, values = (x.double() for x in s["cache"])
        for x, new in ((keys, out[1]), (values, s["v"].double())):
            flat = x[0].transpose(1, 2).reshape(-1, c["kv_heads"], c["hd"])  # row = slot
            flat[s["slots"].long()[s["slots"] >= 0]] = new[s["slots"] >= 0]
            x[0] = flat.view(-1, 16, c["kv_heads"], c["hd"]).transpose(1, 2)
        return [out[0], keys, values]
    if c["kind"] == "moe":
        x = s["x"].double()
        z = x @ s["router"].double().t()
        p = torch.sigmoid(z) if c["score"] == "sigmoid" else torch.softmax(z, -1)
        pick = torch.topk(p if s["favour"] is None else p + s["favour"].double(), c["k"], dim=-1)[1]
        w = p.gather(1, pick)
        w = w / w.sum(-1, keepdim=True)
        out = s["residual"].double()
        for e in torch.unique(pick).tolist():  # (fp64 copies of one expert at a time)
            row, slot = (pick == e).nonzero(as_tuple=True)
            h = torch.nn.functional.silu(x[row] @ s["gate"][e].double().t()) * (x[row] @ s["up"][e].double().t())
            out.index_add_(0, row, w[row, slot][:, None] * (h @ s["down"][e].double().t()))
        return {"ids": None, "weights": w, "out": out}
    start, history, tokens = s["start"].tolist(), s["history"], s["tokens"].long()
    x = s["logits"].double()
    for b in range(c["n"]):
        for r in range(start[b], start[b + 1]):
            if c["hist"]:
                before, size = int(s["prompt_len"][b]), int(s["history_len"][b])
                if s["masks"] is None:
                    path = torch.arange(r - start[b] + 1, device="cuda")
                else:
                    i = torch.arange(start[b + 1] - start[b], device="cuda")
                    path = i[(s["masks"][r, i // 64] >> (i % 64)) & 1 == 1]
                count = torch.bincount(torch.cat([history[b, before:size].long(), tokens[start[b] + path]]), minlength=c["vocab"])
                known = torch.bincount(history[b, :before].long(), minlength=c["vocab"]) + count > 0
                again, once, often = (float(p[b]) for p in s["said"])
                x[r, known] = torch.where(x[r, known] > 0, x[r, known] / again, x[r, known] * again)
                x[r] -= often * count + once * (count > 0)
            if c["bias"] and int(s["bias_of"][b]) >= 0:
                x[r] += s["bias"][int(s["bias_of"][b])].double()
            if c["masks"] and int(s["allowed_of"][r]) >= 0:
                word = s["allowed"][int(s["allowed_of"][r])]
                bits = (word[:, None] >> torch.arange(32, device="cuda") & 1).flatten()[:c["vocab"]]
                x[r, bits == 0] = -math.inf
    if c["kind"] == "adjust":
        return x
    top = torch.topk(x, min(c["k"], c["vocab"]), dim=-1)[0]
    total = torch.logsumexp(x, -1)
    return {"best": None, "logprob": torch.where(top == -math.inf, top, top - total[:, None]), "total": total}
