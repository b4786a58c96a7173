"""ssd_tree_attention on the GPU against plain numpy in 64 bits
(tests/tree_reference.py), and a round of all the tree operators.
"""
import math

import numpy as np
import pytest

import tree_reference as ref
from test_gpu_tree_ops import TYPES, dev, ints, random_parents

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ssd():
    import paper_2309_08168_gb300 as m
    return m


class Case:
    """A batch over a paged cache.  What no row may see is NaN: positions behind a request's last, pages of nobody."""

    def __init__(self, rng, kind, heads, kv, hd, page, lens, counts, masks="tree", words=None, apart=False, q_scale=1.5, extra_rows=2, layers=1):
        self.heads, self.kv, self.hd, self.page, self.kind = heads, kv, hd, page, kind
        self.lens, counts = np.array(lens, np.int32), np.array(counts)
        self.row_start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.n_rows, self.max_rows = int(self.row_start[-1]) + extra_rows, int(counts.max())
        total = np.maximum(self.lens, 0).astype(np.int64) + counts
        need = -(-total // page)
        width = int(max(1, need.max())) + 1
        n_pages = int(need.sum()) + 2
        perm, at = rng.permutation(n_pages), 0
        self.table = np.full((len(lens), width), -1, np.int32)
        for b in range(len(lens)):
            self.table[b, :need[b]] = perm[at:at + need[b]]
            at += need[b]
        t = torch.float16 if kind == "f32" else TYPES[kind]
        shape = (layers, n_pages, page, kv, hd) if apart else (layers, n_pages, kv, page, hd)
        self.k, self.v = (torch.full(shape, float("nan"), dtype=t, device="cuda") for _ in range(2))
        if apart:
            self.k, self.v = self.k.transpose(2, 3), self.v.transpose(2, 3)
        for b in range(len(lens)):
            x = np.arange(total[b])
            p, o = (torch.from_numpy(i).cuda() for i in (self.table[b, x // page].astype(np.int64), x % page))
            for c in (self.k, self.v):
                c[layers - 1, p, :, o] = torch.from_numpy(rng.standard_normal((len(x), kv, hd)).astype(np.float32)).cuda().to(t)
        self.q = torch.from_numpy((q_scale * rng.standard_normal((self.n_rows, heads, hd))).astype(np.float32)).cuda().to(TYPES[kind])
        self.masks = None
        if masks is not None:
            self.words = words or -(-max(1, self.max_rows) // 64)
            parents = random_parents(rng, counts, masks)
            m = np.zeros((self.n_rows, self.words), np.uint64)
            for b, n in enumerate(counts):
                seen = []
                for i in range(n):
                    p = parents[self.row_start[b] + i]
                    seen.append((1 << i) | (seen[p] if p >= 0 else 0))
                    for w in range(self.words):
                        m[self.row_start[b] + i, w] = (seen[i] >> (64 * w)) & (2**64 - 1)
            self.masks = m.view(np.int64)

    def run(self, ssd, scale=None, status=None, workspace=None, stream=None, layer=None, out=None):
        kv = ssd.PagedKV(self.k, self.v)
        b = ssd.TreeBatch(dev(self.row_start), dev(self.lens), dev(self.table), self.n_rows, self.max_rows)
        if out is None:
            out = torch.full(self.q.shape, 77.0, dtype=self.q.dtype, device="cuda")
        if workspace is None:
            workspace = torch.full((ssd.ssd_tree_attention_workspace(kv),), 255, dtype=torch.uint8, device="cuda")
        layer = self.k.shape[0] - 1 if layer is None else layer
        ssd.ssd_tree_attention(b, kv, layer, self.q, dev(self.masks) if self.masks is not None else None, scale or 1 / math.sqrt(self.hd), out, workspace, status,
                               torch.cuda.current_stream().cuda_stream if stream is None else stream)
        return out

    def want(self, scale=None):
        k, v = (c[-1].float().cpu().numpy() for c in (self.k, self.v))
        return ref.attention(self.q.double().cpu().numpy(), k, v, self.row_start, self.lens, self.table, self.page, self.masks, scale or 1 / math.sqrt(self.hd))

    def check(self, out, scale=None):
        want, written, (vmax, smax, count) = self.want(scale)
        got = out.double().cpu().numpy()
        assert (got[~written] == 77).all()
        # a score's products enter with 2^-22 (fp32 rows: fp16 pairs of q) and are summed in fp32 in hd / 16 + 4 steps that
        # round or truncate (2^-22 each, of the sum of |products|); the exponential adds 2^-20; a weight enters the second
        # product with 2^-21 (fp32 rows, pairs) or half a step of its type, the sums of weights and outputs in steps of 2^-22
        # for every 16 positions, and 16 for joining parts; then one rounding to the rows' type
        d = smax * (2.0**-22 * (self.hd / 16 + 4 + 1)) + 2.0**-20
        p = {"f32": 2.0**-21, "f16": 2.0**-11, "bf16": 2.0**-8}[self.kind]
        tol = vmax * (2 * np.expm1(d) + 2 * p + 2 * 2.0**-22 * (count / 16 + 20))
        tol = tol[..., None] + np.abs(want) * {"f32": 2.0**-24, "f16": 2.0**-11, "bf16": 2.0**-8}[self.kind] * 1.01 + (2.0**-25 if self.kind == "f16" else 0)
        err = np.where(written[:, None, None], np.abs(got - want), 0)
        assert np.isfinite(got).all()
        assert (err <= tol).all(), ((err / tol).max(), np.unravel_index(np.argmax(err / tol), err.shape))


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,kv,page,lens,counts,masks,apart", [
    (4, 4, 16, [37], [5], "tree", False),
    (1, 1, 16, [0], [1], "tree", False),  # nothing cached: a root sees itself
    (2, 1, 16, [0, 1, 63, 64, 65], [1, 1, 1, 1, 1], None, False),  # single tokens around a tile
    (3, 3, 48, [127, 128, 129, 0], [4, 64, 65, 2], "tree", True),
    (8, 1, 64, [300, -1, 5, 70], [9, 3, 0, 17], "tree", False),  # ended, empty
    (10, 2, 80, [200, 90], [33, 7], "chain", True),  # groups of 5
    (14, 2, 16, [515], [37], "star", False),  # groups of 7: rows end inside a tile
    (6, 6, 256, [1000, 3], [16, 17], "tree", False),
    (4, 2, 32, [40, 700], [130, 100], "tree", False),  # three mask words
    (2, 2, 16, [100, 33], [200, 300], None, False),  # prompt chunks
    (64, 1, 16, [77], [3], "tree", False),  # one KV head for all
    (200, 1, 16, [130], [2], "tree", False),  # a node's heads in two tiles
    (3, 1, 16, [700, 20], [150, 60], None, False),  # chains whose nodes end inside a tile
])
def test_attention(ssd, kind, hd, heads, kv, page, lens, counts, masks, apart):
    c = Case(np.random.default_rng(heads * 100 + page), kind, heads, kv, hd, page, lens, counts, masks, apart=apart)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = c.run(ssd, status=status)
    torch.cuda.synchronize()
    c.check(out)
    assert int(status) == 0
    assert torch.equal(out, c.run(ssd))  # the same bits again


@pytest.mark.parametrize("kind,heads,kv,lens,counts", [("f32", 2, 2, [6000], [1]), ("f16", 8, 1, [20001], [3]), ("bf16", 4, 2, [3000, 9, 7000], [20, 1, 64]),
                                                       ("f32", 4, 4, [2500] + [20] * 40, [3] * 41),
                                                       ("bf16", 4, 2, [5, -1, 130] * 500, [3, 0, 2] * 500)])
def test_attention_along_a_long_cache(ssd, kind, heads, kv, lens, counts):
    c = Case(np.random.default_rng(len(lens) + heads), kind, heads, kv, 128, 64, lens, counts)
    c.check(c.run(ssd))


@pytest.mark.parametrize("kind,heads,kv,hd,page,n,rows,length,masks", [
    ("f32", 32, 32, 128, 16, 24, 1, 1500, None), ("f16", 32, 8, 128, 48, 20, 17, 1300, "tree"), ("bf16", 16, 2, 64, 64, 30, 40, 900, "tree"),
    ("f32", 16, 16, 128, 16, 3, 700, 600, None), ("bf16", 32, 4, 128, 32, 2, 900, 300, None), ("f32", 24, 8, 64, 80, 50, 9, 700, "tree")])
def test_many_items(ssd, kind, heads, kv, hd, page, n, rows, length, masks):
    """More items than CTAs: ranges with several items, against 64-bit sums on the GPU; the same bits every time."""
    rng = np.random.default_rng(heads + n)
    counts, lens = rng.integers((rows + 1) // 2, rows + 1, n), rng.integers(length // 6, length + 1, n)
    c = Case(rng, kind, heads, kv, hd, page, lens, counts, masks)
    out = c.run(ssd)
    g, scale = heads // kv, 1 / math.sqrt(hd)
    for b in range(n):
        r0, r1, total = int(c.row_start[b]), int(c.row_start[b + 1]), int(c.lens[b] + counts[b])
        x = np.arange(total)
        p, o = torch.from_numpy(c.table[b, x // page].astype(np.int64)).cuda(), torch.from_numpy(x % page).cuda()
        k, v = (t[0, p, :, o].double() for t in (c.k, c.v))
        seen = torch.ones(r1 - r0, total, dtype=torch.bool, device="cuda")
        if masks is None:
            seen = torch.from_numpy(x[None] <= int(c.lens[b]) + np.arange(r1 - r0)[:, None]).cuda()
        else:
            j = torch.arange(r1 - r0, device="cuda")
            seen[:, int(c.lens[b]):] = (dev(c.masks)[r0:r1][:, j // 64] >> (j % 64)) & 1 == 1
        q = c.q[r0:r1].double().unflatten(1, (kv, g))
        s = torch.einsum("tkgd,pkd->tkgp", q, k) * scale
        sums = torch.einsum("tkgd,pkd->tkgp", q.abs(), k.abs()).amax(-1) * scale
        w = torch.softmax(s.masked_fill(~seen[:, None, None], -math.inf), -1)
        want = torch.einsum("tkgp,pkd->tkgd", w, v).flatten(1, 2)
        # as in Case.check
        d = sums.flatten(1, 2)[..., None] * (2.0**-22 * (hd / 16 + 5)) + 2.0**-20
        pe = {"f32": 2.0**-21, "f16": 2.0**-11, "bf16": 2.0**-8}[kind]
        tol = v.abs().max() * (2 * torch.expm1(d) + 2 * pe + 2 * 2.0**-22 * (total / 16 + 20)) + want.abs() * {"f32": 2.0**-24}.get(kind, pe) * 1.01 + 2.0**-25
        assert bool(((out[r0:r1].double() - want).abs() <= tol).all())
    for _ in range(10):
        assert torch.equal(out, c.run(ssd))


def test_the_largest_row_count_only_chooses_the_tile(ssd):
    for heads, kv, counts, said in ((4, 4, [70, 3], 1), (8, 2, [40, 60], 2), (2, 2, [3, 1], 500)):
        c = Case(np.random.default_rng(14), "f16", heads, kv, 128, 16, [300, 40], counts)
        c.max_rows = said
        c.check(c.run(ssd))


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hd,page", [(64, 16), (64, 48), (128, 16), (128, 80)])
@pytest.mark.parametrize("group,said", [(1, 1), (2, 1), (1, 2)])
def test_tiles_of_few_rows(ssd, kind, hd, page, group, said):
    """Trees and chains as tiles of one row or two (heads of a node, or nodes): rows that see nothing, nodes of NaN that some rows do not see, pages outside
    the cache, items of less than a block, of more than a warp looks up at once, and more items than CTAs."""
    rng = np.random.default_rng(30 + hd + group)
    lens, counts = [0, 1, 15, 127, 130, 700, -1, 18000, 31], [3, 1, 17, 1, 70, 2, 0, 1, 33]
    for masks in ("star", None):
        c = Case(rng, kind, 2 * group, 2, hd, page, lens, counts, masks)
        c.max_rows = said
        if masks:
            c.masks[1] = 0  # of a request with nothing cached
        clean = c.run(ssd)
        c.check(clean)
        assert masks is None or (clean[1] == 0).all()
        # the 20th node of request 4: seen by itself (star) or by the rows from it on (chain)
        x, hit = 130 + 20, int(c.row_start[4]) + 20
        for t in (c.k, c.v):
            t[0, int(c.table[4, x // page]), :, x % page] = float("nan")
        out, hits = c.run(ssd), [hit] if masks else range(hit, int(c.row_start[5]))
        others = [r for r in range(c.n_rows) if r not in hits]
        assert torch.equal(out[others], clean[others]) and out[list(hits)].isnan().all()
        c.table[5, 2], c.table[7, 3] = -1, 10**6
        c.row_start, c.lens, c.table = c.row_start[5:].copy(), c.lens[5:], np.ascontiguousarray(c.table[5:])  # without the NaN's request
        c.check(c.run(ssd))


@pytest.mark.parametrize("kind,kv,group,hd,n,length", [("f32", 32, 1, 128, 24, 900), ("f16", 24, 2, 128, 20, 1300), ("bf16", 40, 1, 64, 30, 500), ("f32", 16, 2, 64, 40, 70),
                                                      ("f16", 2, 1, 64, 1500, 40)])
def test_single_tokens_of_many_requests(ssd, kind, kv, group, hd, n, length):
    rng = np.random.default_rng(40 + n)
    c = Case(rng, kind, kv * group, kv, hd, 16, rng.integers(0, length + 1, n), [1] * n, None)
    out = c.run(ssd)
    c.check(out)
    for _ in range(10):
        assert torch.equal(out, c.run(ssd))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_values_that_are_not_finite_in_a_prompt(ssd, kind):
    """A NaN in the values of one position of a chain reaches the rows from it on, an infinity in one dim of another
    position only that dim; the rows before do not change."""
    c = Case(np.random.default_rng(15), kind, 2, 1, 64, 16, [70], [400], None)
    clean = c.run(ssd)
    for node, dim, what in ((300, slice(None), float("nan")), (130, 9, float("inf"))):
        x = 70 + node
        c.v[0, int(c.table[0, x // 16]), :, x % 16, dim] = what
    out = c.run(ssd)
    assert torch.equal(out[:130], clean[:130])
    keep = [d for d in range(64) if d != 9]
    assert torch.equal(out[130:300][:, :, keep], clean[130:300][:, :, keep]) and not out[130:300, :, 9].isfinite().any()
    assert out[300:400].isnan().all()


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_rows_that_see_nothing_are_zero(ssd, kind):
    c = Case(np.random.default_rng(1), kind, 4, 2, 64, 16, [0, 30], [7, 70])
    c.masks[2] = c.masks[5] = 0  # of the request with nothing cached
    c.masks[10] = 0              # of the other one: its cached positions only
    out = c.run(ssd)
    c.check(out)
    assert (out[[2, 5]] == 0).all()


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv,counts", [(4, 4, [9, 5]), (16, 2, [40, 30])])
def test_what_a_row_does_not_see_does_not_matter(ssd, kind, heads, kv, counts):
    """NaN and infinities in the keys and values of single nodes reach the rows that see them, and no others."""
    c = Case(np.random.default_rng(2), kind, heads, kv, 128, 16, [50, 70], counts, "star")
    clean = c.run(ssd)
    bad = {0: (3, float("nan"), None), 1: (4, None, float("inf"))}
    for b, (node, knew, vnew) in bad.items():
        x = int(c.lens[b]) + node
        page, at = int(c.table[b, x // 16]), x % 16
        if knew is not None:
            c.k[0, page, :, at] = knew
            c.v[0, page, :, at, ::2] = knew
        if vnew is not None:
            c.v[0, page, :, at, 5] = vnew
    out = c.run(ssd)
    hit = [int(c.row_start[b]) + node for b, (node, _, _) in bad.items()]
    rest = [r for r in range(int(c.row_start[-1])) if r not in hit]
    assert torch.equal(out[rest], clean[rest])
    assert out[hit[0]].isnan().all()
    assert (out[hit[1], :, 5] == float("inf")).all()
    keep = [d for d in range(128) if d != 5]
    assert torch.equal(out[hit[1]][:, keep], clean[hit[1]][:, keep])


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv,hd,rows", [(8, 8, 128, 25), (8, 8, 64, 32), (32, 8, 128, 12), (16, 8, 64, 40)])
def test_a_large_key_that_a_row_does_not_see(ssd, kind, heads, kv, hd, rows):
    """A node of an item's second unit, most of which every row sees, has a key of fifty times the size: the row of it moves to its
    score, the others of its warp keep their bits (their reference and what they have summed up).  With 320 items most lie in one
    CTA's range."""
    n, rng = 40, np.random.default_rng(60 + rows)
    lens = rng.integers(200, 257 - rows, n)
    c = Case(rng, kind, heads, kv, hd, 16, lens, [rows] * n, "star")
    clean = c.run(ssd)
    node = rng.integers(1, rows, n)
    x = torch.from_numpy(lens + node)
    c.k[0, torch.from_numpy(c.table[np.arange(n), x // 16].astype(np.int64)).cuda(), :, (x % 16).cuda()] *= 50
    out = c.run(ssd)
    hit = (np.arange(n) * rows + node).tolist()
    rest = [r for r in range(n * rows) if r not in hit]
    assert torch.equal(out[rest], clean[rest]) and not torch.equal(out[hit], clean[hit])
    c.check(out)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [3, 40])
def test_scores_of_minus_infinity_have_no_weight(ssd, kind, rows):
    """Keys of -inf in one dim, against positive queries there; a row all of whose scores are -inf is zero."""
    c = Case(np.random.default_rng(3), kind, 4, 2, 64, 16, [0, 0], [rows, rows], None)
    c.q[:, :, 7] = c.q[:, :, 7].abs() + 0.5
    for b in (0, 1):
        for x in ([0, 2] if b == 0 else [0, 1]):  # request 1: the first two rows see only such keys
            c.k[0, int(c.table[b, 0]), :, x, 7] = -float("inf")
    out = c.run(ssd)
    first = int(c.row_start[1])
    assert (out[0] == 0).all() and (out[first:first + 2] == 0).all()
    c.check(out)


def test_large_scores_and_values(ssd):
    """Peaked rows (one position has all the weight), fp32 queries far outside fp16's range and far below it."""
    for q_scale, scale in ((40.0, None), (1e6, 1e-6), (1e-9, 1e9), (1e-3, None)):
        c = Case(np.random.default_rng(4), "f32", 4, 2, 64, 16, [200, 3], [6, 40], q_scale=q_scale)
        c.check(c.run(ssd, scale), scale)


def test_pages_outside_the_cache_read_as_zeros(ssd):
    c = Case(np.random.default_rng(5), "f16", 4, 2, 64, 16, [100], [20])
    c.table[0, 2], c.table[0, 4] = -1, 10**6
    c.check(c.run(ssd))


def test_table_too_narrow(ssd):
    """Positions that the table does not hold are not seen; the call says so."""
    for rows in (3, 30):
        c = Case(np.random.default_rng(6), "f32", 4, 2, 64, 16, [60], [rows])
        c.table = np.ascontiguousarray(c.table[:, :2])
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = c.run(ssd, status=status)
        c.check(out)
        assert int(status) == ssd.SSD_STATUS_TABLE


@pytest.mark.parametrize("heads,kv,said", [(8, 2, 70), (2, 2, 1), (4, 2, 1)])
@pytest.mark.parametrize("words", [1, 2])
def test_more_nodes_than_mask_bits(ssd, heads, kv, said, words):
    """Nodes behind the masks' bits are seen by no row, and the call says so; one that has ended does
    not count."""
    n = 64 * words
    for lens, counts, bits in (([40, 9, -1], [3, n + 6, 0], 4), ([40, 9, -1], [3, n, n + 9], 0)):
        c = Case(np.random.default_rng(72), "f16", heads, kv, 64, 16, lens, counts, words=words)
        c.max_rows = said
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        c.check(c.run(ssd, status=status))
        assert int(status) == bits == (ssd.SSD_STATUS_PARENT if bits else 0)


def test_broken_row_starts_stay_inside(ssd):
    for rows in (2, 60):
        c = Case(np.random.default_rng(7), "f16", 4, 2, 64, 16, [60, 20], [rows, rows], extra_rows=0)
        c.row_start = np.array([-4, 2 * rows + 90, 1], np.int32)
        guard = torch.full((c.n_rows + 64, 4, 64), 77.0, dtype=torch.float16, device="cuda")
        c.masks[:] = -1
        c.run(ssd, out=guard[32:32 + c.n_rows])
        torch.cuda.synchronize()
        assert (guard[:32] == 77).all() and (guard[32 + c.n_rows:] == 77).all()


def test_layers_and_strided_rows(ssd):
    """The layer asked for is read; q and out may be parts of wider rows."""
    c = Case(np.random.default_rng(8), "bf16", 4, 2, 128, 48, [90, 10], [30, 4], layers=3, apart=True)
    n, w = c.n_rows, 4 * 128
    wide, res = torch.zeros(n, w + 64, dtype=torch.bfloat16, device="cuda"), torch.full((n, w + 8), 77.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 64:] = c.q.reshape(n, w)
    c.q = wide[:, 64:].unflatten(1, (4, 128))
    out = c.run(ssd, out=res[:, :w].unflatten(1, (4, 128)))
    c.check(out)
    assert (res[:, w:] == 77).all()


def test_on_another_stream_and_in_graphs_that_share_a_workspace(ssd):
    a = Case(np.random.default_rng(9), "f32", 8, 2, 128, 16, [900, 40], [9, 3])
    b = Case(np.random.default_rng(10), "f16", 16, 2, 64, 16, [500, 700], [60, 64])
    want = [a.run(ssd), b.run(ssd)]
    ws = torch.full((ssd.ssd_tree_attention_workspace(ssd.PagedKV(a.k, a.v)),), 255, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = a.run(ssd, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(out, want[0])
    graphs, outs = [], []
    for c in (a, b):
        kv, o = ssd.PagedKV(c.k, c.v), torch.full(c.q.shape, 77.0, dtype=c.q.dtype, device="cuda")
        bt, m = ssd.TreeBatch(dev(c.row_start), dev(c.lens), dev(c.table), c.n_rows, c.max_rows), dev(c.masks)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ssd.ssd_tree_attention(bt, kv, 0, c.q, m, 1 / math.sqrt(c.hd), o, ws, None, torch.cuda.current_stream().cuda_stream)
        graphs.append((g, bt, m, kv))
        outs.append(o)
    for _ in range(3):
        for (g, *_), o in zip(graphs, outs):
            o.fill_(77.0)
            g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_two_calls_at_once(ssd):
    """Two streams, a workspace each: neither call changes the other's bits."""
    cases = [Case(np.random.default_rng(20 + i), kind, heads, kv, 128, 16, lens, counts)
             for i, (kind, heads, kv, lens, counts) in enumerate((("f32", 16, 4, [2000] * 6, [9] * 6), ("bf16", 32, 4, [1500] * 5, [33] * 5)))]
    want = [c.run(ssd) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    spaces = [torch.empty(ssd.ssd_tree_attention_workspace(ssd.PagedKV(c.k, c.v)), dtype=torch.uint8, device="cuda") for c in cases]
    calls, outs = [], []
    for c in cases:
        kv, o = ssd.PagedKV(c.k, c.v), torch.full(c.q.shape, 77.0, dtype=c.q.dtype, device="cuda")
        outs.append(o)
        calls.append((ssd.TreeBatch(dev(c.row_start), dev(c.lens), dev(c.table), c.n_rows, c.max_rows), kv, 0, c.q, dev(c.masks), 1 / math.sqrt(c.hd), o))
    torch.cuda.synchronize()
    for _ in range(20):
        for a, ws, st in zip(calls, spaces, streams):
            ssd.ssd_tree_attention(*a, ws, None, st.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_a_captured_call_follows_the_lengths(ssd):
    """Lengths, starts and tables are read when the graph runs."""
    c = Case(np.random.default_rng(11), "f32", 4, 2, 64, 16, [900, 800], [9, 3])
    kv, ws = ssd.PagedKV(c.k, c.v), torch.empty(ssd.ssd_tree_attention_workspace(ssd.PagedKV(c.k, c.v)), dtype=torch.uint8, device="cuda")
    lens, m = dev(c.lens), dev(c.masks)
    bt, o = ssd.TreeBatch(dev(c.row_start), lens, dev(c.table), c.n_rows, c.max_rows), torch.full(c.q.shape, 77.0, device="cuda")
    c.run(ssd)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ssd.ssd_tree_attention(bt, kv, 0, c.q, m, 0.125, o, ws, None, torch.cuda.current_stream().cuda_stream)
    for new in ([900, 800], [3, 500], [0, 64], [-1, 1]):
        c.lens = np.array(new, np.int32)
        lens.copy_(torch.from_numpy(c.lens))
        o.fill_(77.0)
        g.replay()
        c.check(o, 0.125)


@pytest.mark.parametrize("kind,heads,kv", [("f32", 4, 4), ("bf16", 6, 3)])
def test_captured_single_tokens(ssd, kind, heads, kv):
    """A decoding step as a graph: every replay sees what the lengths hold then."""
    c = Case(np.random.default_rng(21), kind, heads, kv, 128, 32, [700, 300, 40, 0], [1] * 4, None)
    cache, lens, out = ssd.PagedKV(c.k, c.v), dev(c.lens), torch.full(c.q.shape, 77.0, dtype=c.q.dtype, device="cuda")
    ws = torch.empty(ssd.ssd_tree_attention_workspace(cache), dtype=torch.uint8, device="cuda")
    bt, g = ssd.TreeBatch(dev(c.row_start), lens, dev(c.table), c.n_rows, 1), torch.cuda.CUDAGraph()
    c.run(ssd)
    with torch.cuda.graph(g):
        ssd.ssd_tree_attention(bt, cache, 0, c.q, None, 128**-0.5, out, ws, None, torch.cuda.current_stream().cuda_stream)
    for new in ([700, 300, 40, 0], [129, 127, -1, 0], [0, 0, 0, 0], [-1, -1, -1, -1], [690, 1, 33, -1]):
        c.lens = np.array(new, np.int32)
        lens.copy_(torch.from_numpy(c.lens))
        out.fill_(77.0)
        g.replay()
        c.check(out)


def test_empty_rounds_and_empty_masks(ssd):
    """A round without rows is a call that does nothing, with masks as without; masks of no words are refused, not taken for none."""
    c = Case(np.random.default_rng(73), "f16", 4, 2, 64, 16, [9, 30], [0, 0], extra_rows=0)
    c.max_rows = 1
    assert c.masks.shape == (0, 1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert c.run(ssd, status=status).shape == (0, 4, 64)
    c.masks = None
    c.run(ssd, status=status)
    c = Case(np.random.default_rng(74), "f16", 4, 2, 64, 16, [9, 30], [3, 2])
    c.masks = c.masks[:, :0]
    with pytest.raises(ssd.SSDError):
        c.run(ssd, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0


def test_tensors_elsewhere_are_refused(ssd):
    c = Case(np.random.default_rng(12), "f32", 2, 2, 64, 16, [9], [2])
    c.q = c.q.cpu()
    with pytest.raises(ssd.SSDError):
        c.run(ssd)
    with pytest.raises(ssd.SSDError):
        ssd.PagedKV(c.k.cpu(), c.v.cpu())
    host = torch.zeros(64, dtype=torch.int32)
    b = ssd.ssd_batch(1, 1, 1, 1, host.data_ptr(), host.data_ptr(), host.data_ptr())
    assert ssd.lib.ssd_tree_plan(b, 16, 10, None, *[host.data_ptr() + 16 * i for i in range(7)], None, 0, None, None) == ssd.SSD_ERR_INVALID_ARG
    assert "current device" in ssd.ssd_last_error()


@pytest.mark.parametrize("heads,kv,rows", [(2, 2, 1), (4, 2, 9)])
def test_offsets_beyond_32_bits(ssd, heads, kv, rows):
    """Pages and layers more than 2^32 bytes apart: the cache's rows, the attention over them and the moved rows are those
    of a compact cache."""
    page, hd, n_pages, layers = 16, 64, 3, 2
    far = 2**31 + 64
    big = torch.empty(layers * n_pages * far, dtype=torch.float16, device="cuda")  # 26 GB, of which little is touched
    inner = (2 * page * hd, hd, 1)  # [kv_head][position][dim], K and V one after the other in a head's place
    spread = [big[o:].as_strided((layers, n_pages, kv, page, hd), (n_pages * far, far) + inner) for o in (0, page * hd)]
    small = [torch.zeros(layers, n_pages, kv, page, hd, dtype=torch.float16, device="cuda") for _ in range(2)]
    for t in spread:
        t.zero_()
    table, s = dev(np.array([[2, 0, 1]], np.int32)), torch.cuda.current_stream().cuda_stream
    rope = ssd.ssd_rope_init(hd)
    res = []
    for k, v in (spread, small):
        rng = np.random.default_rng(23)
        cache, out = ssd.PagedKV(k, v), []
        ws = torch.empty(ssd.ssd_tree_attention_workspace(cache), dtype=torch.uint8, device="cuda")
        def step(n, length):
            q, kk, vv = (torch.from_numpy(rng.standard_normal((n, h, hd)).astype(np.float32)).cuda().half() for h in (heads, kv, kv))
            x = np.arange(length, length + n)
            slots = np.array([2, 0, 1])[x // page] * page + x % page
            for layer in range(layers):
                ssd.ssd_rope_kv(cache, layer, rope, q, kk, vv, dev(x.astype(np.int32)), dev(slots.astype(np.int32)), q, s)
            bt = ssd.TreeBatch(dev(np.array([0, n], np.int32)), ints(1).fill_(length), table, n, n)
            o = torch.empty_like(q)
            ssd.ssd_tree_attention(bt, cache, layers - 1, q, None, hd**-0.5, o, ws, None, s)
            return o, bt
        out.append(step(30, 0)[0])
        o, bt = step(rows, 30)
        out.append(o)
        # every draft but the first is right: node 2's chain, as children of the root
        parents = np.array([-1, 0] + [0] * (rows > 2) + list(range(2, rows - 1)), np.int32)[:rows]
        tokens, target = np.arange(rows, dtype=np.int32), np.full(rows, 99, np.int32)
        if rows > 2:
            target[0], target[2:rows - 1] = 2, np.arange(3, rows)
        got = [ints(1) for _ in range(3)] + [ints(rows) for _ in range(2)]
        ssd.ssd_tree_commit(bt, cache, dev(parents), dev(tokens), dev(target), *got, s)
        assert int(got[0]) == max(rows - 2, 0)
        out += [k.clone(), v.clone()]
        res.append(out)
    assert all(torch.equal(x, y) for x, y in zip(*res)) and float(res[1][2][1, 2].abs().sum()) > 0
    del big, spread, cache, t, k, v
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cta", [0, 7, 151])
def test_a_wait_that_gives_up(ssd, kind, cta):
    """A CTA whose keys never come: its waits end after their limit, the call ends and says so, rows of requests that it has no part in are as ever, and so
    are the calls after it."""
    c = Case(np.random.default_rng(70), kind, 8, 4, 128, 16, [700] * 60, [9] * 60)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.full((ssd.ssd_tree_attention_workspace(ssd.PagedKV(c.k, c.v)),), 255, dtype=torch.uint8, device="cuda")
    want = c.run(ssd, status=status, workspace=ws)
    assert int(status) == 0
    ssd.ssd_debug_tree_stall(cta, 0.01)
    out = c.run(ssd, status=status)  # (with a workspace of its own, without an older call's parts)
    assert int(status) == ssd.SSD_STATUS_TIMEOUT
    same = (out == want).flatten(1).all(1)[:int(c.row_start[-1])].view(60, 9).all(1)
    assert 50 <= int(same.sum()) < 60  # (a CTA has 240 items of six units and three more / 152 of them)
    status.zero_()
    assert torch.equal(c.run(ssd, status=status, workspace=ws), want) and int(status) == 0
    ssd.ssd_debug_tree_stall(cta, 0.01)
    ssd.ssd_debug_tree_stall(-1)
    assert torch.equal(c.run(ssd, status=status, workspace=ws), want) and int(status) == 0


def test_tiles_of_few_rows_have_no_waits(ssd):
    """Such a call does not stall."""
    few = Case(np.random.default_rng(71), "f16", 4, 4, 64, 16, [300], [1], None)
    ssd.ssd_debug_tree_stall(0, 0.01)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    few.check(few.run(ssd, status=status))
    assert int(status) == 0
    ssd.ssd_debug_tree_stall(-1)


def test_a_request_without_pages_touches_no_others(ssd):
    """One of two requests gets no page for its round's rows.  With -1 behind the pages that it holds, the rest of the round reads and
    moves nothing of anyone else's, and the other request's round is as it would be alone."""
    rng = np.random.default_rng(75)
    page, n_pages, kv, hd, n = 16, 6, 2, 64, 7
    table, lens = np.array([[3, -1, -1], [0, -1, -1]], np.int32), np.array([12, 14], np.int32)
    parents = np.tile(np.array([-1, 0, 0, 0, 0, 0, 5], np.int32), 2)  # accepted: nodes 5 and 6, which lie in a second page
    tokens, target = np.tile(np.arange(n, dtype=np.int32), 2), np.full(2 * n, 99, np.int32)
    target[[0, n]], target[[5, n + 5]] = 5, 6
    kc, vc = (torch.from_numpy(rng.standard_normal((1, n_pages, kv, page, hd)).astype(np.float32)).cuda().half() for _ in range(2))
    before = kc.clone(), vc.clone()
    cache, ring, ends, held = ssd.PagedKV(kc, vc), dev(np.array([5, 1, 2, 4, -9, -9], np.int32)), torch.tensor([0, 1], device="cuda"), dev(np.array([1, 1], np.int32))
    tb, rows = dev(table), dev(np.array([0, n, 2 * n], np.int32))
    bt = ssd.TreeBatch(rows, dev(lens), tb, 2 * n, n)
    held2, ends2, slots, pos, masks, status = ints(2), torch.zeros_like(ends), ints(2 * n), ints(2 * n), torch.zeros(2 * n, 1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    ssd.ssd_tree_plan(bt, page, n_pages, dev(parents), held, held2, ring, ends, ends2, slots, pos, masks, status, s)
    assert int(status) == ssd.SSD_STATUS_PAGES and tb.cpu().tolist() == [[3, 5, -1], [0, -1, -1]] and (slots[n:] == -1).all()
    q, k, v = (torch.randn(2 * n, h, hd, device="cuda").half() for h in (4, kv, kv))
    ssd.ssd_rope_kv(cache, 0, ssd.ssd_rope_init(hd), q, k, v, pos, slots, q, s)
    out, ws = torch.full_like(q, 77.0), torch.empty(ssd.ssd_tree_attention_workspace(cache), dtype=torch.uint8, device="cuda")
    ssd.ssd_tree_attention(bt, cache, 0, q, masks, 0.125, out, ws, status, s)
    got = [ints(2), ints(2), ints(2), ints(2 * n), ints(2 * n)]
    written = kc.clone(), vc.clone()
    ssd.ssd_tree_commit(bt, cache, dev(parents), dev(tokens), dev(target), *got, s)
    torch.cuda.synchronize()
    assert got[0].cpu().tolist() == [2, 2] and int(got[2][0]) == 15
    for t, w, b in zip((kc, vc), written, before):
        assert torch.equal(t[:, [0, 1, 2, 4]], b[:, [0, 1, 2, 4]])  # the held page of request 1 and those of no one
        assert torch.equal(t[0, 3, :, 13], w[0, 5, :, 1]) and torch.equal(t[0, 3, :, 14], w[0, 5, :, 2])
    alone = ssd.TreeBatch(rows[:2].clone(), dev(lens[:1]), tb[:1].clone(), n, n)
    kc.copy_(written[0])
    vc.copy_(written[1])
    first = torch.empty_like(out[:n])
    ssd.ssd_tree_attention(alone, cache, 0, q[:n], masks[:n].clone(), 0.125, first, ws, status, s)
    assert torch.equal(first, out[:n])


# -- a round of all of them ---------------------------------------------------

@pytest.mark.parametrize("kind,heads,kv,hd,page,tree", [("f32", 4, 2, 64, 16, True), ("f16", 8, 1, 128, 48, True), ("bf16", 4, 4, 64, 16, False)])
def test_rounds_of_a_batch(ssd, kind, heads, kv, hd, page, tree):
    """Prompts, then rounds of drafted trees: plan, rope, attention, commit.  q, k and v of a token follow from the token
    alone; after every round the cache of each request holds its sequence, and the rows' attention is what the
    sequence through their ancestors gives.  Requests end and their pages serve others."""
    rng = np.random.default_rng(13)
    t, ct, n, vocab = TYPES[kind], torch.float16 if kind == "f32" else TYPES[kind], 3, 50
    emb = [torch.from_numpy(rng.standard_normal((vocab, h, hd)).astype(np.float32)).cuda().to(t) for h in (heads, kv, kv)]
    n_pages, width = 3 * (-(-130 // page)) , -(-130 // page)
    kc, vc = (torch.full((1, n_pages, kv, page, hd), float("nan"), dtype=ct, device="cuda") for _ in range(2))
    cache, rope = ssd.PagedKV(kc, vc), ssd.ssd_rope_init(hd, 1e4)
    f = ref.frequencies(hd)
    ring = torch.arange(n_pages, dtype=torch.int32, device="cuda")
    ends, held, table = torch.tensor([0, n_pages], device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), ints(n, width)
    lens = torch.zeros(n, dtype=torch.int32, device="cuda")
    ws = torch.empty(ssd.ssd_tree_attention_workspace(cache), dtype=torch.uint8, device="cuda")
    seqs = [rng.integers(0, vocab, int(k)).tolist() for k in (33, 1, 20)]  # the last token of each is not cached
    s = torch.cuda.current_stream().cuda_stream
    for step in range(9):
        prompt = step == 0
        if step == 5:  # request 1 ends; the next round starts another one in its place
            lens[1] = -1
        counts, parents, tokens = [], [], []
        for b in range(n):
            if int(lens[b]) < 0:
                counts.append(0)
                continue
            c = len(seqs[b]) if prompt or int(lens[b]) == 0 else int(rng.integers(1, 13))
            counts.append(c)
            if prompt or int(lens[b]) == 0 or not tree:
                parents += range(-1, c - 1)
            else:
                parents += [-1] + [int(rng.integers(0, i)) for i in range(1, c)]
            tokens += seqs[b] if prompt or int(lens[b]) == 0 else [seqs[b][-1]] + rng.integers(0, 3, c - 1).tolist()
        row_start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        rows = int(row_start[-1])
        words = -(-max(counts) // 64) if tree else 0
        pt, tk = dev(np.array(parents, np.int32)) if tree else None, dev(np.array(tokens, np.int32))
        bt = ssd.TreeBatch(dev(row_start), lens, table, rows, max(counts))
        held2, ends2, slots, pos = ints(n), torch.zeros_like(ends), ints(rows), ints(rows)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        masks = torch.zeros(rows, words, dtype=torch.int64, device="cuda") if tree else None
        ssd.ssd_tree_plan(bt, page, n_pages, pt, held, held2, ring, ends, ends2, slots, pos, masks, status, s)
        q, k, v = (e[tk.long()] for e in emb)
        turned, out = torch.empty_like(q), torch.empty_like(q)
        ssd.ssd_rope_kv(cache, 0, rope, q, k, v, pos, slots, turned, s)
        ssd.ssd_tree_attention(bt, cache, 0, turned, masks, hd**-0.5, out, ws, status, s)
        # what each row's own sequence gives
        assert int(status) == 0
        for b in range(n):
            for i in range(counts[b]):
                r = int(row_start[b]) + i
                line, x = [], i
                while x >= 0:
                    line.insert(0, tokens[row_start[b] + x])
                    x = parents[row_start[b] + x]
                line = (seqs[b][:int(lens[b])] if not prompt else []) + line
                assert int(pos[r]) == len(line) - 1
                kk = torch.from_numpy(ref.rope(emb[1][line].double().cpu().numpy(), np.arange(len(line)), f, False)).to(ct).double().numpy()
                vv = emb[2][line].to(ct).double().cpu().numpy()
                qq = ref.rope(emb[0][line[-1:]].double().cpu().numpy(), [len(line) - 1], f, False)[0]
                g = heads // kv
                sc = np.einsum("hd,phd->hp", qq, np.repeat(kk, g, 1)) * hd**-0.5
                w = np.exp(sc - sc.max(1, keepdims=True))
                o = np.einsum("hp,phd->hd", w / w.sum(1, keepdims=True), np.repeat(vv, g, 1))
                # keys (and in 16 bits queries, weights, outputs) rounded to their type
                tol = {"f32": 8 * 2.0**-11, "f16": 12 * 2.0**-11, "bf16": 12 * 2.0**-8}[kind] * np.abs(vv).max()
                assert np.abs(out[r].double().cpu().numpy() - o).max() <= tol
        # the target's choices: the drafts mostly, then something else
        target = rng.integers(0, 3, rows).astype(np.int32)
        acc, nxt, new = ints(n), ints(n), ints(n)
        path, emitted = ints(rows), ints(rows)
        if prompt or any(counts[b] and int(lens[b]) == 0 for b in range(n)):  # prompts are taken whole
            target = np.concatenate([np.array(tokens[1:] + [2], np.int32)])
            for b in range(n):
                if counts[b]:
                    target[row_start[b + 1] - 1] = 2
        ssd.ssd_tree_commit(bt, cache, pt, tk, dev(target), acc, nxt, new, path, emitted, s)
        torch.cuda.synchronize()
        for b in range(n):
            if not counts[b]:
                continue
            a = int(acc[b])
            got = emitted[int(row_start[b]):int(row_start[b]) + a + 1].cpu().tolist()
            if prompt or int(lens[b]) == 0:
                seqs[b] = seqs[b] + got[len(seqs[b]) - 1:] if a >= len(seqs[b]) - 1 else seqs[b][:a + 1] + got[-1:]
            else:
                seqs[b] += got
            assert int(new[b]) == len(seqs[b]) - 1 and got[-1] == int(nxt[b])
            x = np.arange(int(new[b]))
            tb = table[b].cpu().numpy()
            have = kc[0][torch.from_numpy(tb[x // page].astype(np.int64)), :, torch.from_numpy(x % page)].double().cpu().numpy()
            line = seqs[b][:-1]
            full = ref.rope(emb[1][line].double().cpu().numpy(), x, f, False)
            assert np.abs(have - full).max() <= {"f32": 1.01 * 2.0**-11, "f16": 1.01 * 2.0**-11, "bf16": 1.01 * 2.0**-8}[kind] * 2 * np.abs(full).max() + 1e-5
        held, ends = held2, ends2
        lens.copy_(new)
        if step == 5:
            assert int(held[1]) == 0
            lens[1] = 0
            seqs[1] = rng.integers(0, vocab, 7).tolist()
    assert int(ends[1]) > n_pages  # pages came back
