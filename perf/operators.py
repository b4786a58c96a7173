"""The operators for trees of drafted tokens over a paged cache, as they are measured.

Four kinds of case:

  plan    ssd_tree_plan: pages for the requests' new rows, block tables, the rows' slots, positions and ancestor masks
  rope    ssd_rope_kv: queries and keys turned to their positions, keys and values written to their cache rows
  attn    ssd_tree_attention: attention of a batch's rows over the cache, with tree masks or as chains
  commit  ssd_tree_commit: the accepted path of every tree, its keys and values moved behind the prefix

Lengths and row counts of a batch follow from the case alone (the work of a case
has to be known without its inputs); everything else is made from the seed.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_LEFT = -7  # what outputs hold before a call: entries that no row owns keep it


def listed():
    return [
        # the next round of one short request: 5 rows, latency only
        dict(name="plan_one", kind="plan", n=1, rows=5, ctx=37, page=16, tree=True),
        # a full serving batch, trees of 64 nodes, some requests that ended
        dict(name="plan_batch", kind="plan", n=1000, rows=64, ctx=8000, page=16, tree=True),
        # one decoding step of a single request at 7B widths
        dict(name="rope_step", kind="rope", type="f32", heads=32, kv_heads=32, hd=128, n=1, rot=128, pairs="half", scaling="none", far=2000),
        # trees of a batch at 70B widths, far positions, frequencies scaled by parts
        dict(name="rope_tree", kind="rope", type="bf16", heads=64, kv_heads=8, hd=128, n=400, rot=128, pairs="half", scaling="parts", far=120000),
        # a prompt, half of each head rotated in neighbouring pairs
        dict(name="rope_prompt", kind="rope", type="f16", heads=32, kv_heads=32, hd=128, n=8191, rot=64, pairs="neighbours", scaling="linear", far=8190),
        # the smallest verification: 4 drafts after a short prompt
        dict(name="attn_small", kind="attn", type="f32", heads=4, kv_heads=4, hd=64, n=1, rows=5, ctx=37, page=16, tree=True),
        # single tokens of 16 requests at 7B widths, ragged lengths
        dict(name="attn_step", kind="attn", type="f32", heads=32, kv_heads=32, hd=128, n=16, rows=1, ctx=2100, page=16, tree=False),
        # trees of 33 nodes at 70B widths (grouped heads)
        dict(name="attn_tree", kind="attn", type="bf16", heads=64, kv_heads=8, hd=128, n=6, rows=33, ctx=4096, page=64, tree=True),
        # one request with a very long context and a small tree: all of the work lies along the cache
        dict(name="attn_long", kind="attn", type="f16", heads=64, kv_heads=8, hd=128, n=1, rows=9, ctx=100001, page=256, tree=True),
        # chunks of two prompts at 13B widths
        dict(name="attn_chunk", kind="attn", type="f32", heads=40, kv_heads=40, hd=128, n=2, rows=1023, ctx=700, page=48, tree=False),
        # the end of a round of one request
        dict(name="commit_one", kind="commit", type="f16", kv_heads=4, hd=64, layers=4, n=1, rows=9, ctx=60, page=16),
        # and of a batch
        dict(name="commit_batch", kind="commit", type="f16", kv_heads=8, hd=128, layers=32, n=48, rows=64, ctx=100, page=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "rope", "rope", "attn", "attn", "attn", "attn", "commit"])
    page = rng.choice([16, 16, 32, 48, 64, 80, 128, 256])
    if kind == "plan":
        n = _log(rng, 1, 1000)
        tree = rng.random() < 0.7
        return dict(kind=kind, n=n, rows=_log(rng, 1, 250 if n < 80 else 64) if tree else _log(rng, 1, max(1, 60000 // n)), ctx=_log(rng, 1, 8000), page=page, tree=tree)
    hd = rng.choice([64, 128, 128])
    kv = _log(rng, 1, 40)
    group = rng.choice([1, 1, 2, 4, 5, 8])
    if kv * group > 64:
        kv = 64 // group
    typ = rng.choice(["f32", "f16", "bf16"])
    if kind == "rope":
        rot = rng.choice([hd, hd, hd // 2, hd // 4, 48])
        n = _log(rng, 1, min(16000, 80_000_000 // (kv * (group + 2) * hd)))
        return dict(kind=kind, type=typ, heads=kv * group, kv_heads=kv, hd=hd, n=n, rot=rot, pairs=rng.choice(["half", "neighbours"]),
                    scaling=rng.choice(["none", "linear", "parts"]), far=_log(rng, 2, 1000000))
    if kind == "commit":
        rows = _log(rng, 1, 100)
        return dict(kind=kind, type=rng.choice(["f16", "bf16"]), kv_heads=min(kv, 8), hd=hd, layers=rng.randint(1, 32), n=_log(rng, 1, 32), rows=rows,
                    ctx=_log(rng, 1, 100), page=rng.choice([16, 32, 48, 64]))
    tree = rng.random() < 0.6
    while True:
        n = _log(rng, 1, 32)
        rows = _log(rng, 1, 128) if tree else rng.choice([1, _log(rng, 1, 1000)])
        ctx = _log(rng, 1, 60000)
        # at most the cache and the score matrix of the largest listed cases
        if n * (ctx + rows) * kv * hd <= 1e8 and n * rows * kv * group * (ctx + rows) <= 8e7:
            return dict(kind=kind, type=typ, heads=kv * group, kv_heads=kv, hd=hd, n=n, rows=rows, ctx=ctx, page=page, tree=tree)


# -- sizes and inputs -----------------------------------------------------------

def _sizes(c):
    """(lengths, row counts) of the requests; the first is as long as they get.  plan: every 16th request has ended."""
    rng = random.Random(1000 * c["n"] + c["rows"])
    lens = [c["ctx"]] + [rng.randint(c["ctx"] // 8, c["ctx"]) for _ in range(c["n"] - 1)]
    rows = [c["rows"]] + [rng.randint((c["rows"] + 1) // 2, c["rows"]) for _ in range(c["n"] - 1)]
    if c["kind"] == "plan":
        for b in range(15, c["n"], 16):
            lens[b], rows[b] = -1, 0
    return lens, rows


def _need(c, length, rows):
    return -(-(length + rows) // c["page"]) if length >= 0 else 0


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _batch(c):
    """What every batch has: where its requests' rows start, how many positions of each are cached."""
    lens, rows = _sizes(c)
    start = [0]
    for t in rows:
        start.append(start[-1] + t)
    return {"lens": _ints(lens), "start": _ints(start), "n_rows": start[-1], "rows": rows}


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tree_parents(s, g):
    """Random trees, parents before children: the parent of node i lies in [i / 4, i)."""
    node, _ = _nodes(s["start"], s["n_rows"])
    lo = node // 4
    p = lo + (torch.rand(s["n_rows"], device="cuda", generator=g) * (node - lo)).long()
    return torch.where(node == 0, -1, torch.minimum(p, node - 1)).int()


def _nodes(start, n):
    """(index within its request, request) of rows 0 .. n-1."""
    r = torch.arange(n, device=start.device)
    b = torch.searchsorted(start[1:].contiguous(), r.int(), right=True)
    return r - start.long()[b], b


def _reach(parents, node, b, n_requests, width):
    """[request][i][j]: whether node j is node i or above it."""
    m = torch.eye(width, device="cuda").repeat(n_requests, 1, 1)
    has = parents >= 0
    m[b[has], node[has], parents.long()[has]] = 1.0
    for _ in range(max(1, (width - 1).bit_length())):  # (paths of twice the length each time)
        m = ((m @ m) > 0).float()
    return m


def _mask_bits(reach, words):
    """The rows of `reach` as 64-bit words, bit j of word w for node 64 w + j."""
    pad = torch.zeros(*reach.shape[:2], 64 * words, dtype=torch.int64, device="cuda")
    pad[..., : reach.shape[2]] = reach.long()
    return (pad.view(*reach.shape[:2], words, 64) << torch.arange(64, device="cuda")).sum(-1)


def _words(c):
    return -(-c["rows"] // 64) if c["tree"] else 0


def prepare(case, seed):
    s = {"plan": _prepare_plan, "rope": _prepare_rope, "attn": _prepare_attn, "commit": _prepare_commit}[case["kind"]](case, seed)
    return {"case": case, **s}


def _prepare_plan(c, seed):
    g, s = _generator(seed), _batch(c)
    lens, rows = _sizes(c)
    # requests hold the pages of their cached positions; the ended ones still hold some
    held = [_need(c, n, 0) if n >= 0 else 1 + b % 5 for b, n in enumerate(lens)]
    fresh = sum(max(0, _need(c, n, t) - h) for n, t, h in zip(lens, rows, held))
    width = max(max(held), max(_need(c, n, t) for n, t in zip(lens, rows))) + 1
    n_pages = sum(held) + fresh + 8
    perm = torch.randperm(n_pages, generator=g, device="cuda").int()
    held_t = _ints(held)
    first = torch.cumsum(held_t, 0) - held_t
    j = torch.arange(width, device="cuda")
    at = first[:, None] + j
    table = torch.where(j < held_t[:, None], perm[at.clamp(max=n_pages - 1)], torch.full_like(at, _LEFT)).int()
    # the other pages are free: they stand in the ring from `head` on
    free, head = fresh + 8, seed % n_pages
    ring = torch.full((n_pages,), _LEFT, dtype=torch.int32, device="cuda")
    ring[(head + torch.arange(free, device="cuda")) % n_pages] = perm[n_pages - free:]
    s.update(table=table, held=held_t, ring=ring, ends=torch.tensor([head, head + free], device="cuda"), n_pages=n_pages)
    s["parents"] = _tree_parents(s, g) if c["tree"] else None
    n, w = s["n_rows"], _words(c)
    s["out"] = {"held": torch.full_like(held_t, _LEFT), "ends": torch.full_like(s["ends"], _LEFT), "slots": torch.full((n,), _LEFT, dtype=torch.int32, device="cuda"),
                "positions": torch.full((n,), _LEFT, dtype=torch.int32, device="cuda"), "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if c["tree"]:
        s["out"]["masks"] = torch.full((n, w), _LEFT, dtype=torch.int64, device="cuda")
    if own:
        import paper_2309_08168_gb300 as ssd
        s["batch"] = ssd.TreeBatch(s["start"], s["lens"], table, n, c["rows"])
    return s


def _cache(c, n_pages, layers, g):
    """Keys and values [layer][page][kv_head][position][dim]."""
    t = torch.float16 if c["type"] == "f32" else _TYPES[c["type"]]
    return [torch.empty(layers, n_pages, c["kv_heads"], c["page"], c["hd"], dtype=t, device="cuda").normal_(0.0, 1.0, generator=g) for _ in range(2)]


_SCALING = {"none": dict(), "linear": dict(factor=4.0), "parts": dict(factor=8.0, original=4096, slow=1.0, fast=32.0, amplitude=0.1 * math.log(8.0) + 1.0)}


def _prepare_rope(c, seed):
    g, n = _generator(seed), c["n"]
    width = (c["heads"] + 2 * c["kv_heads"]) * c["hd"]
    packed = torch.randn(n, width, device="cuda", generator=g).to(_TYPES[c["type"]])  # the projections' output, q then k then v
    n_pages = -(-n * 5 // 4 // 16) + 1
    cache = _cache(dict(c, page=16), n_pages, 1, g)
    slots = torch.randperm(n_pages * 16, generator=g, device="cuda")[:n].int()
    slots[seed % n] = -1 if n > 1 else slots[0]  # a row that has no place in the cache
    positions = torch.randint(max(1, c["far"] // 2), c["far"] + 1, (n,), generator=g, device="cuda").int()
    q, k, v = packed.split([c["heads"] * c["hd"], c["kv_heads"] * c["hd"], c["kv_heads"] * c["hd"]], 1)
    s = {"q": q.unflatten(1, (c["heads"], c["hd"])), "k": k.unflatten(1, (c["kv_heads"], c["hd"])), "v": v.unflatten(1, (c["kv_heads"], c["hd"])),
         "positions": positions, "slots": slots, "cache": cache, "q_out": torch.empty(n, c["heads"], c["hd"], dtype=packed.dtype, device="cuda")}
    if own:
        import paper_2309_08168_gb300 as ssd
        x = _SCALING[c["scaling"]]
        kind = {"none": ssd.SSD_ROPE_PLAIN, "linear": ssd.SSD_ROPE_LINEAR, "parts": ssd.SSD_ROPE_BY_PARTS}[c["scaling"]]
        s["kv"] = ssd.PagedKV(*cache)
        s["rope"] = ssd.ssd_rope_init(c["rot"], theta=1e4, interleaved=c["pairs"] == "neighbours", scaling=kind, factor=x.get("factor", 1.0),
                                      original_len=x.get("original", 0), slow=x.get("slow", 0.0), fast=x.get("fast", 0.0), amplitude=x.get("amplitude", 1.0))
    return s


def _table(c, g):
    """Every request's pages, anywhere in the cache."""
    lens, rows = _sizes(c)
    need = _ints([_need(c, n, t) for n, t in zip(lens, rows)])
    total, width = sum(_need(c, n, t) for n, t in zip(lens, rows)), max(_need(c, n, t) for n, t in zip(lens, rows))
    perm = torch.randperm(total + 3, generator=g, device="cuda").int()
    j = torch.arange(width, device="cuda")
    at = (torch.cumsum(need, 0) - need)[:, None] + j
    return torch.where(j < need[:, None], perm[at.clamp(max=total)], torch.full_like(at, -1)).int(), total + 3


def _prepare_attn(c, seed):
    g, s = _generator(seed), _batch(c)
    s["table"], n_pages = _table(c, g)
    s["cache"] = _cache(c, n_pages, 1, g)
    s["q"] = (1.5 * torch.randn(s["n_rows"], c["heads"], c["hd"], device="cuda", generator=g)).to(_TYPES[c["type"]])
    s["out"] = torch.empty_like(s["q"])
    s["masks"] = None
    if c["tree"]:
        node, b = _nodes(s["start"], s["n_rows"])
        s["masks"] = _mask_bits(_reach(_tree_parents(s, g), node, b, c["n"], c["rows"]), _words(c))[b, node].contiguous()
    if own:
        import paper_2309_08168_gb300 as ssd
        s["kv"] = ssd.PagedKV(*s["cache"])
        s["batch"] = ssd.TreeBatch(s["start"], s["lens"], s["table"], s["n_rows"], c["rows"])
        s["workspace"] = torch.empty(ssd.ssd_tree_attention_workspace(s["kv"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_commit(c, seed):
    """Every tree holds `wide` chains of drafts below its root, of which the last one is accepted for some steps.
    (`wide` exceeds the accepted steps, so that no row is both moved and written over and a pass can be repeated.)"""
    g, s = _generator(seed), _batch(c)
    s["table"], n_pages = _table(c, g)
    s["cache"] = _cache(c, n_pages, c["layers"], g)
    n = s["n_rows"]
    node, b = _nodes(s["start"], n)
    count = (s["start"][1:] - s["start"][:-1]).long()[b]
    wide = max(1, math.isqrt(max(0, c["rows"] - 1)) + 1)
    s["parents"] = torch.where(node == 0, -1, torch.where(node <= wide, 0, node - wide)).int()
    steps = (torch.rand(c["n"], device="cuda", generator=g) * wide).long()[b]  # accepted at most, if the tree is deep enough
    target = torch.randint(16000, 32000, (n,), generator=g, device="cuda").int()
    tokens = torch.randint(0, 16000, (n,), generator=g, device="cuda").int()
    good = (node > 0) & (node % wide == 0) & (node // wide <= steps) & (node < count)
    above = s["start"].long()[b] + s["parents"].clamp(min=0)
    s["tokens"], s["target"] = torch.where(good, target[above], tokens), target
    one = torch.full((c["n"],), _LEFT, dtype=torch.int32, device="cuda")
    s["out"] = {"accepted": one, "next": one.clone(), "lens": one.clone(), "path": torch.full((n,), _LEFT, dtype=torch.int32, device="cuda"),
                "emitted": torch.full((n,), _LEFT, dtype=torch.int32, device="cuda")}
    if own:
        import paper_2309_08168_gb300 as ssd
        s["kv"] = ssd.PagedKV(*s["cache"])
        s["batch"] = ssd.TreeBatch(s["start"], s["lens"], s["table"], n, c["rows"])
    return s


# -- one pass ---------------------------------------------------------------------

def run(state):
    return {"plan": _run_plan, "rope": _run_rope, "attn": _run_attn, "commit": _run_commit}[state["case"]["kind"]](state["case"], state)


def _run_plan(c, s):
    o = s["out"]
    if own:
        import paper_2309_08168_gb300 as ssd
        ssd.ssd_tree_plan(s["batch"], c["page"], s["n_pages"], s["parents"], s["held"], o["held"], s["ring"], s["ends"], o["ends"], o["slots"], o["positions"],
                          o.get("masks"), o["status"], torch.cuda.current_stream().cuda_stream)
        return dict(o, table=s["table"], ring=s["ring"])
    lens, held, ring, ends, page, n_pages = s["lens"].long(), s["held"].long(), s["ring"], s["ends"], c["page"], s["n_pages"]
    count = (s["start"][1:] - s["start"][:-1]).long()
    live = lens >= 0
    need = torch.where(live, (lens + count + page - 1) // page, 0)
    fits = need <= s["table"].shape[1]
    new = torch.where(live & fits, (need - held).clamp(min=0), 0)
    upto = torch.cumsum(new, 0)
    given = live & fits & ((new == 0) | (upto <= ends[1] - ends[0]))
    new = torch.where(given, new, 0)
    back = torch.where(live, 0, held)
    j = torch.arange(s["table"].shape[1], device="cuda")
    free = ring.long()[(ends[0] + (upto - new)[:, None] + j - held[:, None]) % n_pages]
    table = torch.where(given[:, None] & (j >= held[:, None]) & (j < need[:, None]), free.int(), s["table"])
    to = (ends[1] + (torch.cumsum(back, 0) - back)[:, None] + j) % n_pages
    gone = j < back[:, None]
    ring = ring.index_put((to[gone],), s["table"][gone])
    node, b = _nodes(s["start"], s["n_rows"])
    at = lens[b] + node
    slots = torch.where(given[b], table.long()[b, (at // page).clamp(0, j.numel() - 1)] * page + at % page, -1)
    out = {"held": torch.where(live, held + new, 0).int(), "ends": torch.stack([ends[0] + new.sum(), ends[1] + back.sum()]), "slots": slots.int(),
           "status": (1 * (live & fits & ~given).any() + 2 * (live & ~fits).any()).int().reshape(1), "table": table, "ring": ring}
    if not c["tree"]:
        return dict(out, positions=at.int())
    reach = _reach(s["parents"], node, b, c["n"], c["rows"])
    return dict(out, positions=(lens[b] + reach.sum(-1).long()[b, node] - 1).int(), masks=_mask_bits(reach, _words(c))[b, node])


def _frequencies(c):
    """Radians a position of every rotated pair, in 64 bits."""
    x = _SCALING[c["scaling"]]
    f = 1e4 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda") / c["rot"])
    if c["scaling"] == "linear":
        return f / x["factor"]
    if c["scaling"] == "parts":
        turns = x["original"] * f / (2 * math.pi)  # over the original context
        keep = ((turns - x["slow"]) / (x["fast"] - x["slow"])).clamp(0, 1)
        return f / x["factor"] * (1 - keep) + f * keep
    return f


def _turn(c, x, cos, sin):
    """The first `rot` dims of each head turned by their pairs' angles, in 32 bits."""
    r, h = c["rot"], c["rot"] // 2
    x = x.float()
    if c["pairs"] == "half":
        a, b = x[..., :h], x[..., h:r]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., r:]], -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., r:]], -1)


def _run_rope(c, s):
    if own:
        import paper_2309_08168_gb300 as ssd
        ssd.ssd_rope_kv(s["kv"], 0, s["rope"], s["q"], s["k"], s["v"], s["positions"], s["slots"], s["q_out"], torch.cuda.current_stream().cuda_stream)
        return [s["q_out"], *s["cache"]]
    angle = s["positions"].double()[:, None] * _frequencies(c)
    m = _SCALING[c["scaling"]].get("amplitude", 1.0)
    cos, sin = (m * angle.cos()).float()[:, None], (m * angle.sin()).float()[:, None]
    keys, values = s["cache"]
    has = s["slots"] >= 0
    page, at = s["slots"].long()[has] // 16, s["slots"].long()[has] % 16
    keys[0, page, :, at] = _turn(c, s["k"], cos, sin)[has].to(keys.dtype)
    values[0, page, :, at] = s["v"][has].to(values.dtype)
    return [_turn(c, s["q"], cos, sin).to(s["q"].dtype), keys, values]


def _run_attn(c, s):
    if own:
        import paper_2309_08168_gb300 as ssd
        ssd.ssd_tree_attention(s["batch"], s["kv"], 0, s["q"], s["masks"], 1.0 / math.sqrt(c["hd"]), s["out"], s["workspace"], None,
                               torch.cuda.current_stream().cuda_stream)
        return s["out"]
    n, wide, page = c["n"], c["rows"], c["page"]
    lens, start = s["lens"].long(), s["start"].long()
    longest = s["table"].shape[1] * page
    # every request padded to the longest one: [request][kv head][position][dim]
    rows = s["table"].long().clamp(min=0)
    keys, values = (x[0][rows].transpose(1, 2).reshape(n, c["kv_heads"], longest, c["hd"]).float() for x in s["cache"])
    node = torch.arange(wide, device="cuda")
    row = (start[:-1, None] + node).clamp(max=s["n_rows"] - 1)  # [request][node]
    q = s["q"].float()[row].view(n, wide, c["kv_heads"], -1, c["hd"]).permute(0, 2, 3, 1, 4).reshape(n, c["kv_heads"], -1, c["hd"])
    j = torch.arange(longest, device="cuda") - lens[:, None]  # the node at a position; negative: cached before
    if s["masks"] is None:
        seen = j[:, None] <= node[:, None]
    else:
        word = (j.clamp(0, 64 * s["masks"].shape[1] - 1) // 64)[:, None].expand(n, wide, longest)
        bit = s["masks"][row].gather(2, word) >> (j % 64)[:, None] & 1
        seen = (j[:, None] < 0) | ((bit == 1) & (j[:, None] < wide))
    seen = (seen & (j < (start[1:] - start[:-1])[:, None])[:, None]).repeat(1, c["heads"] // c["kv_heads"], 1)[:, None]
    x = (q @ keys.transpose(2, 3) / math.sqrt(c["hd"])).masked_fill_(~seen, -math.inf)
    x = (x - x.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x @ values) / torch.where(total == 0, 1.0, total)
    o = o.view(n, c["kv_heads"], -1, wide, c["hd"]).permute(0, 3, 1, 2, 4).reshape(n, wide, c["heads"], c["hd"])
    at, b = _nodes(s["start"], s["n_rows"])
    return o[b, at].to(s["q"].dtype)


def _run_commit(c, s):
    o = s["out"]
    if own:
        import paper_2309_08168_gb300 as ssd
        ssd.ssd_tree_commit(s["batch"], s["kv"], s["parents"], s["tokens"], s["target"], o["accepted"], o["next"], o["lens"], o["path"], o["emitted"],
                            torch.cuda.current_stream().cuda_stream)
        return dict(o, k=s["cache"][0], v=s["cache"][1])
    n, page, start, lens = s["n_rows"], c["page"], s["start"].long(), s["lens"].long()
    node, b = _nodes(s["start"], n)
    above = start[b] + s["parents"].clamp(min=0)
    # the lowest of a node's children that carries the node's chosen token, if any
    fits = (s["parents"] >= 0) & (s["tokens"] == s["target"][above])
    child = torch.full((n + 1,), n, device="cuda").scatter_reduce(0, torch.where(fits, above, n), torch.arange(n, device="cuda"), "amin")
    child[n] = n
    # row after 0, 1, 2, .. steps from the root; n: the path has ended
    steps = [start[:-1]]
    for _ in range(c["rows"] - 1):
        steps.append(child[steps[-1]])
    steps = torch.stack(steps, 1)
    on = steps < n
    accepted = on.sum(1) - 1
    last = steps.gather(1, accepted[:, None])[:, 0]
    path, emitted = o["path"].clone(), o["emitted"].clone()
    k = torch.arange(c["rows"], device="cuda").expand_as(steps)
    path[(start[:-1, None] + k)[on]] = (steps - start[:-1, None])[on].int()
    taken = on & (k > 0)
    emitted[(start[:-1, None] + k - 1)[taken]] = s["tokens"][steps[taken]]
    emitted[start[:-1] + accepted] = s["target"][last]
    of = torch.arange(c["n"], device="cuda")[:, None].expand_as(steps)[taken]
    src, dst = lens[of] + (steps - start[:-1, None])[taken], lens[of] + k[taken]
    src, dst = ((s["table"].long()[of, x // page], x % page) for x in (src, dst))
    for x in s["cache"]:
        x[:, dst[0], :, dst[1]] = x[:, src[0], :, src[1]]
    return {"accepted": accepted.int(), "next": s["target"][last], "lens": (lens + 1 + accepted).int(), "path": path, "emitted": emitted, "k": s["cache"][0], "v": s["cache"][1]}


# -- the work of one pass -----------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "rope":
        e = 4 if c["type"] == "f32" else 2
        row = c["hd"] * (e * (2 * c["heads"] + 2 * c["kv_heads"]) + 2 * 2 * c["kv_heads"])
        return {"bytes": float(c["n"] * (row + 8)), "flops": 3.0 * c["n"] * c["rot"] * (c["heads"] + c["kv_heads"])}
    lens, rows = _sizes(c)
    if c["kind"] == "plan":
        held = [_need(c, n, 0) if n >= 0 else 1 + b % 5 for b, n in enumerate(lens)]
        moved = sum(max(0, _need(c, n, t) - h) if n >= 0 else h for n, t, h in zip(lens, rows, held))
        # lengths, starts, pages held (in, out); pages handed over; parents, slots, positions, masks
        return {"bytes": float(16 * c["n"] + 8 * moved + sum(rows) * ((12 + 8 * _words(c)) if c["tree"] else 8) + 32), "flops": 0.0}
    if c["kind"] == "commit":
        wide = max(1, math.isqrt(max(0, c["rows"] - 1)) + 1)
        moved = sum(min((wide - 1) / 2, (t - 1) // wide) for t in rows)  # steps accepted, about
        return {"bytes": float(moved * c["layers"] * c["kv_heads"] * c["hd"] * 2 * 2 * 2 + 12 * sum(rows) + 16 * c["n"]), "flops": 0.0}
    e = 4 if c["type"] == "f32" else 2
    cache = sum(n + t for n, t in zip(lens, rows)) * c["kv_heads"] * c["hd"] * 2 * 2
    seen = sum(t * n + t * (t + 1) / 2 for n, t in zip(lens, rows))  # (a tree's rows see less of its own nodes than a chain's)
    return {"bytes": float(cache + 2 * e * sum(rows) * c["heads"] * c["hd"]), "flops": 4.0 * c["heads"] * c["hd"] * seen}


# -- the same in 64 bits --------------------------------------------------------------

def exact(case, seed):
    c = case
    if c["kind"] == "plan":
        return None  # whole numbers
    s = prepare(case, seed)
    if c["kind"] == "commit":
        start, lens, parents, tokens, target, table = (s[x].tolist() for x in ("start", "lens", "parents", "tokens", "target", "table"))
        k, v = (x.double() for x in s["cache"])
        for b in range(c["n"]):
            at, step, r0 = 0, 0, start[b]
            while True:
                below = [i for i in range(at + 1, start[b + 1] - r0) if parents[r0 + i] == at and tokens[r0 + i] == target[r0 + at]]
                if not below:
                    break
                at, step = below[0], step + 1
                p, q = lens[b] + at, lens[b] + step
                for x in (k, v):
                    x[:, table[b][q // c["page"]], :, q % c["page"]] = x[:, table[b][p // c["page"]], :, p % c["page"]]
        return {"accepted": None, "next": None, "lens": None, "path": None, "emitted": None, "k": k, "v": v}
    if c["kind"] == "rope":
        out = []
        rate = [1e4 ** (-2 * i / c["rot"]) for i in range(c["rot"] // 2)]
        if c["scaling"] == "linear":
            rate = [f / 4 for f in rate]
        if c["scaling"] == "parts":
            keep = [min(1.0, max(0.0, (4096 * f / (2 * math.pi) - 1) / 31)) for f in rate]
            rate = [f * (k + (1 - k) / 8) for f, k in zip(rate, keep)]
        z = torch.polar(torch.tensor(1.0 + (0.1 * math.log(8.0) if c["scaling"] == "parts" else 0.0), dtype=torch.float64, device="cuda"),
                        torch.outer(s["positions"].double(), torch.tensor(rate, dtype=torch.float64, device="cuda")))[:, None]
        for x in (s["q"].double(), s["k"].double()):
            h = c["rot"] // 2
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
    lens, rows = _sizes(c)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group, r0 = c["heads"] // c["kv_heads"], 0
    for b, (length, t) in enumerate(zip(lens, rows)):
        total = length + t
        at = torch.arange(total, device="cuda")
        page = s["table"][b].long()[at // c["page"]]
        keys, values = (x[0, page, :, at % c["page"]].double() for x in s["cache"])  # [position][kv head][dim]
        if s["masks"] is None:
            seen = at[None] <= length + torch.arange(t, device="cuda")[:, None]
        else:
            i = torch.arange(t, device="cuda")
            seen = torch.ones(t, total, dtype=torch.bool, device="cuda")
            seen[:, length:] = (s["masks"][r0: r0 + t][:, i // 64] >> (i % 64)) & 1 == 1
        for h in range(c["kv_heads"]):
            q = s["q"][r0: r0 + t, h * group: (h + 1) * group].double()
            x = torch.einsum("tgd,pd->tgp", q, keys[:, h]) * c["hd"] ** -0.5
            w = torch.softmax(x.masked_fill(~seen[:, None], -math.inf), -1)
            out[r0: r0 + t, h * group: (h + 1) * group] = torch.einsum("tgp,pd->tgd", w, values[:, h])
        r0 += t
    return out
