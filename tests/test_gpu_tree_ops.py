"""ssd_tree_plan, ssd_rope_kv and ssd_tree_commit on the GPU against plain numpy
(tests/tree_reference.py).  Whole numbers and moved values are equal; rotated
values are held to a bound from their roundings.
"""
import numpy as np
import pytest

import tree_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

LEFT = -7


@pytest.fixture(scope="module")
def ssd():
    import paper_2309_08168_gb300 as m
    return m


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def ints(n, width=None):
    return torch.full((n,) if width is None else (n, width), LEFT, dtype=torch.int32, device="cuda")


# -- plan ---------------------------------------------------------------------

def random_parents(rng, counts, kind):
    out = []
    for n in counts:
        for i in range(n):
            if kind == "chain" or i == 0:
                out.append(i - 1)
            elif kind == "star":
                out.append(0)
            elif kind == "roots":
                out.append(-1)
            else:
                out.append(int(rng.integers(max(0, i - 6), i)) if rng.random() < 0.9 else -1)
    return np.array(out, np.int32)


def run_plan(ssd, row_start, lens, parents, table, held, ring, ends, page, n_rows, words, times=1):
    n = len(lens)
    t = {"table": dev(table), "ring": dev(ring), "held": dev(held), "ends": dev(ends)}
    o = {"held": ints(n), "ends": torch.zeros(2, dtype=torch.int64, device="cuda"), "slots": ints(n_rows), "positions": ints(n_rows),
         "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    masks = torch.full((n_rows, words), LEFT, dtype=torch.int64, device="cuda") if words else None
    b = ssd.TreeBatch(dev(row_start), dev(lens), t["table"], n_rows, int(max(1, np.diff(row_start).max())))
    for _ in range(times):
        ssd.ssd_tree_plan(b, page, len(ring), dev(parents) if parents is not None else None, t["held"], o["held"], t["ring"], t["ends"], o["ends"],
                          o["slots"], o["positions"], masks, o["status"], torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    got = {k: v.cpu().numpy() for k, v in o.items()}
    got |= {"table": t["table"].cpu().numpy(), "ring": t["ring"].cpu().numpy(), "masks": None if masks is None else masks.cpu().numpy()}
    got["status"] = int(got["status"][0])
    return got


def same_plan(got, want):
    for k in want:
        if want[k] is None:
            assert got[k] is None
        else:
            assert np.array_equal(got[k], want[k]), (k, got[k], want[k])


def plan_case(rng, n, most_rows, most_len, page, kind, words, spare=5, ended=0.2, extra_rows=3, width=None):
    counts = rng.integers(0, most_rows + 1, n)
    lens = rng.integers(0, most_len + 1, n).astype(np.int32)
    lens[rng.random(n) < ended] = -1
    need = np.where(lens >= 0, -(-(lens.astype(np.int64) + counts) // page), 0)
    held = np.where(lens >= 0, -(-lens.astype(np.int64) // page) + (rng.random(n) < 0.2), rng.integers(0, 4, n))
    wide = int(max(need.max(), held.max())) + 1
    n_pages = int(held.sum() + np.maximum(need - held, 0).sum()) + spare + 1
    perm = rng.permutation(n_pages).astype(np.int32)
    table, at = np.full((n, wide), -9, np.int32), 0
    for b in range(n):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    head = int(rng.integers(0, 1 << 40))
    free = n_pages - at
    ring = np.full(n_pages, -9, np.int32)
    ring[(head + np.arange(free)) % n_pages] = perm[at:]
    row_start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    parents = random_parents(rng, counts, kind) if words else None
    n_rows = int(row_start[-1]) + extra_rows
    if parents is not None:
        parents = np.concatenate([parents, np.full(extra_rows, -1, np.int32)])
    if width is not None:
        table = np.ascontiguousarray(np.concatenate([table, np.full((n, width), -9, np.int32)], 1)[:, :width])
        held = np.minimum(held, width)
    return row_start, lens, parents, table, held.astype(np.int32), ring, np.array([head, head + free]), page, n_rows, words


@pytest.mark.parametrize("n,rows,length,page,kind,words", [
    (1, 1, 0, 16, "tree", 1), (1, 5, 37, 16, "tree", 1), (3, 64, 100, 16, "tree", 1), (7, 65, 100, 48, "tree", 2), (5, 200, 40, 64, "tree", 4),
    (2, 256, 40, 16, "chain", 4), (2, 256, 1000, 256, "star", 4), (2, 130, 10, 16, "roots", 3), (4, 300, 70, 16, "chain", 0), (300, 9, 60, 16, "tree", 1),
    (1500, 3, 200, 16, "tree", 1), (4096, 1, 33, 16, "none", 0), (2, 3000, 5, 80, "none", 0), (1, 40000, 7, 48, "none", 0), (5, 0, 90, 16, "tree", 1)])
def test_plan(ssd, n, rows, length, page, kind, words):
    rng = np.random.default_rng(n * 7 + rows)
    c = plan_case(rng, n, rows, length, page, kind, words)
    same_plan(run_plan(ssd, *c, times=2), ref.plan(*c[:7], c[7], len(c[5]), c[8], c[9]))


def test_plan_without_rows(ssd):
    """Only pages: ended requests give theirs back."""
    rng = np.random.default_rng(2)
    c = list(plan_case(rng, 6, 0, 90, 16, "tree", 1, ended=0.5, extra_rows=0))
    c[9] = 1
    got = run_plan(ssd, *c)
    want = ref.plan(*c[:7], c[7], len(c[5]), c[8], c[9])
    for k in ("table", "ring", "held", "ends"):
        assert np.array_equal(got[k], want[k]), k


def test_plan_short_of_pages(ssd):
    """Requests in order until the first that does not get all; those that need none go on, the others keep theirs."""
    rng = np.random.default_rng(3)
    for spare in (-1, -7, -40):
        c = list(plan_case(rng, 40, 30, 100, 16, "tree", 1))
        c[6] = np.array([c[6][0], max(c[6][0], c[6][1] + spare - 6)])
        want = ref.plan(*c[:7], c[7], len(c[5]), c[8], c[9])
        assert want["status"] == 1
        same_plan(run_plan(ssd, *c), want)


def test_plan_with_a_narrow_table(ssd):
    rng = np.random.default_rng(4)
    c = plan_case(rng, 30, 30, 100, 16, "tree", 1, width=4)
    want = ref.plan(*c[:7], c[7], len(c[5]), c[8], c[9])
    assert want["status"] == 2
    same_plan(run_plan(ssd, *c), want)


def test_plan_bad_parents_are_roots(ssd):
    rng = np.random.default_rng(5)
    c = plan_case(rng, 4, 70, 50, 16, "tree", 1, ended=0.0)  # more than 64 nodes for one word
    c[2][::5] = 1000
    c[2][3::7] = -5
    want = ref.plan(*c[:7], c[7], len(c[5]), c[8], c[9])
    assert want["status"] == 4
    same_plan(run_plan(ssd, *c), want)


def test_plan_with_broken_row_starts_stays_inside(ssd):
    """Starts beyond the rows or in the wrong order own no rows outside the tensors."""
    rng = np.random.default_rng(6)
    c = list(plan_case(rng, 3, 8, 50, 16, "tree", 1, ended=0.0, extra_rows=0))
    n = c[8]
    guard = torch.full((n + 64,), LEFT, dtype=torch.int32, device="cuda")
    table = dev(c[3])
    b = ssd.TreeBatch(dev(np.array([-5, n + 50, 2, n + 60], np.int32)), dev(c[1]), table, n, 8)
    slots = guard[32:32 + n]
    o = ints(3), torch.zeros(2, dtype=torch.int64, device="cuda"), ints(n), torch.zeros(n, 1, dtype=torch.int64, device="cuda")
    ssd.ssd_tree_plan(b, 16, len(c[5]), dev(c[2]), dev(c[4]), o[0], dev(c[5]), dev(c[6]), o[1], slots, o[2], o[3], None, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    g = guard.cpu().numpy()
    assert (g[:32] == LEFT).all() and (g[32 + n:] == LEFT).all()


# -- rope ---------------------------------------------------------------------

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# half a step of a rounding, relative to the value
HALF = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}


def rope_close(got, want, x, dtype, amplitude):
    """fp32: cosine and sine are off by 2^-24 of a turn times 2 pi (3.8e-7) plus sincospif's and the amplitude's
    rounding (3 steps of 2^-24); two products and a sum round once each: 3 * 2^-24.  Then one rounding to the type
    (fp16: at least half of its smallest step, 2^-25)."""
    big = amplitude * 2 * np.abs(x).max(axis=-1, keepdims=True)
    tol = big * (3.8e-7 + 6 * 2.0**-24) + np.abs(want) * HALF[dtype] * 1.01 + (2.0**-25 if dtype == torch.float16 else 0.0)
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), (err - tol).max()


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,heads,kv,hd,rot,inter,page,scaling,far", [
    (1, 4, 4, 64, 64, False, 16, {}, 40), (5, 6, 2, 64, 16, True, 48, {}, 4000), (33, 5, 5, 128, 128, False, 16, dict(scaling=1, factor=4.0), 30000),
    (3, 64, 8, 128, 128, True, 64, dict(scaling=2, factor=8.0, original_len=4096, slow=1.0, fast=32.0, amplitude=1.25), 2**31 - 2),
    (300, 7, 1, 128, 48, False, 256, {}, 1000000), (2, 3, 3, 64, 32, False, 16, {}, 1), (700, 2, 2, 64, 64, True, 16, {}, 5000000)])
def test_rope(ssd, kind, n, heads, kv, hd, rot, inter, page, scaling, far):
    rng = np.random.default_rng(n + heads)
    t = TYPES[kind]
    ct = torch.float16 if kind == "f32" else t
    n_pages, layers = -(-n // page) + 2, 2
    # q, k and v are parts of one row, with a gap behind it; the cache has its heads next to a position's in odd cases
    width = (heads + 2 * kv) * hd + 16
    x = torch.from_numpy(rng.standard_normal((n, width)).astype(np.float32)).cuda().to(t)
    q, k, v = (p.unflatten(1, (-1, hd)) for p in x[:, :width - 16].split([heads * hd, kv * hd, kv * hd], 1))
    if n % 2:
        shape = (layers, n_pages, page, kv, hd)
        kc, vc = (torch.full(shape, float("nan"), dtype=ct, device="cuda").transpose(2, 3) for _ in range(2))
    else:
        kc, vc = (torch.full((layers, n_pages, kv, page, hd), float("nan"), dtype=ct, device="cuda") for _ in range(2))
    slots = rng.permutation(n_pages * page)[:n].astype(np.int32)
    if n > 4:
        slots[1], slots[2], slots[4] = -1, n_pages * page, 2**31 - 1  # not in the cache
    positions = np.concatenate([[far], rng.integers(0, far + 1, n - 1)]).astype(np.int32)
    out = torch.full((n, heads * hd + 8), float("nan"), dtype=t, device="cuda")
    r = ssd.ssd_rope_init(rot, 1e4, inter, **scaling)
    ssd.ssd_rope_kv(ssd.PagedKV(kc, vc), 1, r, q, k, v, dev(positions), dev(slots), out[:, :heads * hd].unflatten(1, (heads, hd)),
                    torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    f = ref.frequencies(rot, 1e4, scaling.get("scaling", 0), scaling.get("factor", 1.0), scaling.get("original_len", 0.0), scaling.get("slow", 1.0),
                        scaling.get("fast", 32.0))
    amp = scaling.get("amplitude", 1.0)
    qn, kn, vn = (p.double().cpu().numpy() for p in (q, k, v))
    rope_close(out[:, :heads * hd].reshape(n, heads, hd), ref.rope(qn, positions, f, inter, amp), qn, t, amp)
    assert out[:, heads * hd:].isnan().all()
    ok = (slots >= 0) & (slots < n_pages * page)
    at = torch.from_numpy(slots[ok].astype(np.int64)).cuda()
    rope_close(kc[1, at // page, :, at % page], ref.rope(kn, positions, f, inter, amp)[ok], kn[ok], ct, amp)
    assert torch.equal(vc[1, at // page, :, at % page], v[torch.from_numpy(ok).cuda()].to(ct))
    # nothing else was written
    kc[1, at // page, :, at % page] = float("nan")
    vc[1, at // page, :, at % page] = float("nan")
    assert kc.isnan().all() and vc.isnan().all()


def test_rope_of_no_rows(ssd):
    kc, vc = (torch.full((1, 1, 2, 16, 64), 3.0, dtype=torch.float16, device="cuda") for _ in range(2))
    for q, k, v in (([torch.empty(0, h, 64, device="cuda") for h in (4, 2, 2)]), [torch.empty(5, h, 64, device="cuda").transpose(0, 1)[:, :0].transpose(0, 1) for h in (4, 2, 2)]):
        none = torch.empty(0, dtype=torch.int32, device="cuda")
        ssd.ssd_rope_kv(ssd.PagedKV(kc, vc), 0, ssd.ssd_rope_init(64), q, k, v, none, none, torch.empty_like(q), torch.cuda.current_stream().cuda_stream)
    assert (kc == 3).all() and (vc == 3).all()


def test_rope_in_place_and_repeated_slots(ssd):
    """q_out in q's place; two rows with one slot: the cache holds one of them."""
    t = torch.float32
    q, k, v = (torch.randn(4, 2, 64, device="cuda") for _ in range(3))
    kc, vc = (torch.zeros(1, 1, 2, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    pos, slots = dev(np.array([5, 6, 7, 8], np.int32)), dev(np.array([3, 3, 0, 1], np.int32))
    want = torch.empty_like(q)
    s = torch.cuda.current_stream().cuda_stream
    r = ssd.ssd_rope_init(64)
    ssd.ssd_rope_kv(ssd.PagedKV(kc, vc), 0, r, q, k, v, pos, slots, want, s)
    got = q.clone()
    ssd.ssd_rope_kv(ssd.PagedKV(kc, vc), 0, r, got, k, v, pos, slots, got, s)
    assert torch.equal(got, want)
    assert any(torch.equal(vc[0, 0, :, 3], v[i].half()) for i in (0, 1)) and t == q.dtype


def test_rope_infinite_and_large_values(ssd):
    """fp32 keys beyond fp16's range become infinite in the cache, NaN stays NaN, each only in its own pair."""
    k = torch.zeros(1, 1, 64, device="cuda")
    k[0, 0, 3], k[0, 0, 40] = 1e6, float("nan")
    v = torch.full((1, 1, 64), -1e6, device="cuda")
    kc, vc = (torch.zeros(1, 1, 1, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    q = torch.zeros(1, 1, 64, device="cuda")
    ssd.ssd_rope_kv(ssd.PagedKV(kc, vc), 0, ssd.ssd_rope_init(64), q, k, v, dev(np.zeros(1, np.int32)), dev(np.zeros(1, np.int32)), torch.empty_like(q),
                    torch.cuda.current_stream().cuda_stream)
    row = kc[0, 0, 0, 0]
    assert row[3] == float("inf") and row[40].isnan() and row[8].isnan()
    rest = torch.ones(64, dtype=torch.bool, device="cuda")
    rest[[3, 35, 40, 8]] = False
    assert (row[rest] == 0).all() and (vc[0, 0, 0, 0] == -float("inf")).all()


# -- commit -------------------------------------------------------------------

@pytest.mark.parametrize("n,rows,layers,kv,hd,page,length,tree", [
    (1, 1, 1, 1, 64, 16, 0, True), (1, 9, 4, 4, 64, 16, 60, True), (6, 40, 3, 5, 128, 48, 100, True), (3, 256, 2, 2, 64, 16, 30, True), (2, 300, 1, 1, 128, 64, 17, False),
    (5, 20, 2, 3, 64, 16, 40, False), (90, 12, 1, 2, 64, 16, 30, True)])
def test_commit(ssd, n, rows, layers, kv, hd, page, length, tree):
    rng = np.random.default_rng(n * 3 + rows)
    counts = rng.integers(max(0, rows - 8), rows + 1, n)
    counts[0] = rows
    lens = rng.integers(0, length + 1, n).astype(np.int32)
    if n > 3:
        lens[2], counts[3] = -1, 0
    row_start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    n_rows = int(row_start[-1]) + 2
    parents = np.concatenate([random_parents(rng, counts, "tree"), [-1, -1]]).astype(np.int32) if tree else None
    # few different tokens: long paths, siblings with the same token
    tokens, target = (rng.integers(0, 2, n_rows).astype(np.int32) for _ in range(2))
    if not tree:
        target[:-1] = np.where(rng.random(n_rows - 1) < 0.95, tokens[1:], 9)
    need = -(-(np.maximum(lens, 0).astype(np.int64) + counts) // page)
    width = int(need.max())
    perm, at = rng.permutation(int(need.sum()) + 1), 0
    table = np.full((n, width), -1, np.int32)
    for b in range(n):
        table[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
    t = torch.float16 if rows % 2 else torch.bfloat16
    kc, vc = (torch.randn(layers, at + 1, kv, page, hd, device="cuda").to(t) for _ in range(2))
    acc, nxt, new, path, emitted, moves = ref.commit(row_start, lens, table, page, parents, tokens, target, n_rows)
    want = [kc.clone(), vc.clone()]
    for x in want:
        for b, src, dst in moves:
            x[:, table[b, dst // page], :, dst % page] = x[:, table[b, src // page], :, src % page].clone()
    o = [ints(n), ints(n), ints(n), ints(n_rows), ints(n_rows)]
    bt = ssd.TreeBatch(dev(row_start), dev(lens), dev(table), n_rows, rows)
    d = [dev(parents) if tree else None, dev(tokens), dev(target)]
    s = torch.cuda.current_stream().cuda_stream
    ssd.ssd_tree_commit(bt, None, *d, *o, s)  # tokens only
    first = [x.clone() for x in o]
    ssd.ssd_tree_commit(bt, ssd.PagedKV(kc, vc), *d, *o, s)
    torch.cuda.synchronize()
    for got, again, x in zip(o, first, (acc, nxt, new, path, emitted)):
        assert np.array_equal(got.cpu().numpy(), x) and torch.equal(got, again)
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])
    assert acc.max() > 1 or n == 1


def test_commit_with_pages_outside_the_cache(ssd):
    """Rows whose pages are not the cache's are not moved and nothing outside is touched."""
    table = np.array([[0, 7, -1]], np.int32)
    kc, vc = (torch.randn(1, 2, 1, 16, 64, device="cuda").half() for _ in range(2))
    want = kc.clone()
    n = 40
    parents = np.array([-1] + [0] * 38 + [38], np.int32)
    tokens = np.arange(n, dtype=np.int32)
    target = np.zeros(n, np.int32)
    target[0], target[38] = 38, 39
    o = [ints(1), ints(1), ints(1), ints(n), ints(n)]
    ssd.ssd_tree_commit(ssd.TreeBatch(dev(np.array([0, n], np.int32)), dev(np.array([3], np.int32)), dev(table), n, n), ssd.PagedKV(kc, vc), dev(parents), dev(tokens),
                        dev(target), *o, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(kc, want) and int(o[0]) == 2 and int(o[2]) == 6
