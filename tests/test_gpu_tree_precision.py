"""How exact ssd_tree_attention is on the GPU, against sums in 64 bits: the norm of the error relative to the
result's.  (A bound for every element, as in tests/test_gpu_tree_attention.py, has to allow for the worst case, which
is hundreds of times what a whole result may be off by.)
"""
import math

import numpy as np
import pytest

from test_gpu_tree_ops import TYPES, dev, random_parents

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ssd():
    import paper_2309_08168_gb300 as m
    return m


def shared_pages(ssd, kind, heads, kv, hd, n, rows, length, masks, mean=0.0, spread=1.0, page=64, steps=()):
    """Attention of n requests of `rows` rows that all see the same `length` cached positions (one table for all, so that
    many long items take little memory).  Values are around `mean` to twice that, by dim; from
    each position of `steps` on, scores are larger by 6.  Returns the result, it in 64 bits, and that rounded to the type."""
    g = torch.Generator(device="cuda").manual_seed(heads + length)
    t = TYPES[kind]
    total = length + rows
    pages = -(-total // page)
    k, v = (torch.randn(1, pages, kv, page, hd, device="cuda", generator=g) for _ in range(2))
    if steps:
        x = torch.arange(pages * page, device="cuda").view(pages, 1, page)
        k[0, ..., 0] = sum((x >= at) * 6.0 * math.sqrt(hd) / 8.0 for at in steps)
    k, v = (x.to(torch.float16 if kind == "f32" else t) for x in (k, spread * v + mean * (1 + torch.rand(kv, 1, hd, device="cuda", generator=g))))
    q = (1.5 * torch.randn(n * rows, heads, hd, device="cuda", generator=g)).to(t)
    if steps:
        q[..., 0] = 8.0
    seen, m = torch.ones(rows, total, dtype=torch.bool, device="cuda"), None
    if masks is None:
        seen[:, length:] = torch.tril(seen[:, length:])
    else:
        parents, own = random_parents(np.random.default_rng(rows), [rows], masks), np.eye(rows, dtype=bool)
        for i in range(rows):
            if parents[i] >= 0:
                own[i] |= own[parents[i]]
        seen[:, length:] = dev(own)
        bits = [sum(1 << j for j in range(rows) if own[i, j]) for i in range(rows)]
        words = np.array([[(b >> (64 * w)) & (2**64 - 1) for w in range(-(-rows // 64))] for b in bits], np.uint64)
        m = dev(np.tile(words.view(np.int64), (n, 1)))
    cache = ssd.PagedKV(k, v)
    i32 = dict(dtype=torch.int32, device="cuda")
    bt = ssd.TreeBatch(torch.arange(n + 1, **i32) * rows, torch.full((n,), length, **i32), torch.arange(pages, **i32).repeat(n, 1), n * rows, rows)
    out, status = torch.empty_like(q), torch.zeros(1, **i32)
    ws = torch.empty(ssd.ssd_tree_attention_workspace(cache), dtype=torch.uint8, device="cuda")
    ssd.ssd_tree_attention(bt, cache, 0, q, m, 1 / math.sqrt(hd), out, ws, status, torch.cuda.current_stream().cuda_stream)
    keys, values = (x[0].transpose(0, 1).reshape(kv, -1, hd)[:, :total].double() for x in (k, v))
    want = torch.empty(n * rows, heads, hd, dtype=torch.float64, device="cuda")
    group = heads // kv
    for r0 in range(0, n * rows, rows):
        for h in range(kv):
            x = torch.einsum("tgd,pd->tgp", q[r0:r0 + rows, h * group:(h + 1) * group].double(), keys[h]) / math.sqrt(hd)
            w = torch.softmax(x.masked_fill_(~seen[:, None], -math.inf), -1)
            want[r0:r0 + rows, h * group:(h + 1) * group] = torch.einsum("tgp,pd->tgd", w, values[h])
    assert int(status) == 0
    return out.double(), want, want.to(t).double()


# tiles of 128 rows that are full or almost empty, more rows than one tile, tiles of one and two rows; with 160 items and more,
# nearly every one lies in one CTA's range
FORMS = [(64, 8, 128, 20, 9, 4200, "tree"), (16, 8, 64, 20, 5, 6000, "tree"), (8, 8, 128, 20, 150, 4100, None), (32, 8, 128, 20, 1, 4500, None),
         (8, 8, 128, 20, 1, 4500, None), (16, 8, 64, 20, 1, 9000, None), (8, 1, 128, 3, 33, 20000, "tree")]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_norm_of_the_error(ssd, kind, form):
    """fp32 rows: 2e-6 at any length (ssd_ops.h: 1e-6).  16-bit rows: what rounding the exact result to the type makes of it (norm r).
    Weights in pairs are off by 2^-22 (fp16) or 2^-17 (bf16, 8e-6) each, scores by some 1e-6, and errors that do not
    depend on each other add in squares: bf16 r = 1.7e-3, fp16 r = 2.1e-4, so 1.00003 r and less; 1.05 r leaves room for the
    sample.  (Weights rounded to the type once would make 1.4 r.)"""
    got, want, rounded = shared_pages(ssd, kind, *form)
    err, r = float((got - want).norm() / want.norm()), float((rounded - want).norm() / want.norm())
    assert err <= (2e-6 if kind == "f32" else 1.05 * r), (err, r)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form", [(8, 8, 128, 20, 3, 100000, "tree"), (8, 8, 64, 20, 3, 100000, "tree"), (8, 8, 128, 20, 40, 30000, None), (8, 8, 128, 20, 1, 60000, None),
                                  (16, 8, 64, 20, 1, 60000, None), (64, 8, 128, 20, 9, 4097, "tree"), (16, 16, 128, 10, 4, 8192, None)], ids=str)
def test_results_do_not_drift(ssd, kind, form):
    """Values of one sign, whole requests in one CTA's range: the mean of the signed error.  What the tensor cores cut off at every step is always
    towards zero, so it grows with the positions that are added in one accumulator: 6e-4 at 100000.  Bounds: an eleventh of fp16's half
    step (2^-11) however long the cache is; for fp32 rows 2e-6."""
    got, want, rounded = shared_pages(ssd, kind, *form, mean=1.0, spread=0.25)
    drift = float(((got - rounded) * want).sum() / (want * want).sum())
    assert abs(drift) <= (2e-6 if kind == "f32" else 4.3e-5), drift


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form,steps", [((8, 8, 128, 20, 40, 9000, "tree"), (3072, 6100, 6208)), ((64, 8, 128, 20, 9, 7000, "tree"), (2944, 3072, 6144, 6300)),
                                        ((16, 8, 64, 20, 30, 9300, None), (1, 3071, 9216)), ((16, 16, 128, 12, 1, 9000, None), (3072, 8000))], ids=str)
def test_references_that_move(ssd, kind, form, steps):
    """Scores rise by 6 (2^8.7) at and around the ends of what is summed up in one accumulator, so that what was summed before has to be
    multiplied there (left out, it would be off by 2^8.7 in weight).  16-bit rows: as in test_norm_of_the_error.  fp32 rows: |scale q k| adds up to S = 6
    a step and 1.5 * 0.64 * hd^0.5 for the other dims; q enters with 2^-22 of it, and the 2 hd / 16 sums of a score are cut at
    2^-23 of S each; a weight is off by as much, and so is the result."""
    got, want, rounded = shared_pages(ssd, kind, *form, steps=steps)
    err, r = float((got - want).norm() / want.norm()), float((rounded - want).norm() / want.norm())
    hd = form[2]
    size = 6 * len(steps) + 0.96 * math.sqrt(hd)
    assert err <= (size * (2.0**-22 + hd / 8 * 2.0**-23) if kind == "f32" else 1.05 * r), (err, r)
