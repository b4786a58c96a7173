"""ssd_logits_choose on the GPU in the variants of large rounds, and masks at the border of what is taken as a list.  Plain numpy."""
import numpy as np
import pytest

import test_gpu_step_logits as logits

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ssd():
    import paper_2309_08168_gb300 as m
    return m


@pytest.mark.parametrize("k", [1, 5])
@pytest.mark.parametrize("typ,vocab,pad", [("f16", 9000, 0), ("bf16", 9000, 0), ("f32", 9000, 0), ("bf16", 9001, 0), ("f16", 20004, 4)])
@pytest.mark.parametrize("hist,masks", [(0, 0), (60, 0), (60, 9)])
def test_biases_of_large_rounds(ssd, k, typ, vocab, pad, hist, masks):
    """400 rows: more CTAs than two an SM take, with biases that lie on 16 bytes where the logits do and that do not."""
    c = logits.Case(50, typ, vocab, None, n=400, hist=hist, few=200, tokens=False, bias=3, masks=masks, pad=pad)
    logits.check(ssd, c, k, want_adjust=False)


@pytest.mark.parametrize("k", [1, 6])
@pytest.mark.parametrize("vocab,n", [(2049, 3), (8185, 320), (50000, 4)])
def test_masks_that_leave_just_an_eighth(ssd, k, vocab, n):
    """A slice is as many tokens as a multiple of 64 of CTAs take; masks leave an eighth of one in its first tokens, and some fewer
    and more, whichever way the row is cut (1, 2, 4 or 8 slices)."""
    counts = []
    for parts in (1, 2, 4, 8):
        s = ((vocab + 7 + parts - 1) // parts + 63) // 64 * 64
        counts += [s // 8 - 1, s // 8, s // 8 + 1]
    c = logits.Case(51, "f32", vocab, None, n=n, hist=40, few=vocab, tokens=False, bias=2, masks=len(counts))
    rng = np.random.default_rng(vocab + k)
    bits = np.zeros((len(counts), -(-vocab // 32) * 32), bool)
    for i, m in enumerate(counts):
        bits[i, rng.permutation(min(vocab, 8 * (counts[i // 3 * 3 + 1]) - 16))[:m]] = True  # (all in the row's first slice)
    c.r["allowed"] = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
    c.r["allowed_of"] = (np.arange(n) % len(counts)).astype(np.int32)
    logits.check(ssd, c, k, want_adjust=False)
    if n < len(counts):
        for first in range(n, len(counts), n):
            c.r["allowed_of"] = ((first + np.arange(n)) % len(counts)).astype(np.int32)
            logits.check(ssd, c, k, want_adjust=False)


@pytest.mark.parametrize("k", [1, 4])
@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_nan_counts_as_minus_infinity(ssd, typ, k):
    """Never chosen, and left out of the row's logsumexp; with masks and without."""
    c = logits.Case(52, typ, 4001, None, n=6, tokens=False, masks=4)
    c.logits[0, ::3] = float("nan")
    c.logits[1, 5] = float("nan")
    c.logits[2] = float("nan")
    c.logits[3, :4000] = float("nan")
    c.logits[4, 17], c.logits[4, 18] = float("nan"), float("inf")
    c.logits[5, 7], c.logits[5, 8:] = float("nan"), -float("inf")
    c.host = c.logits.float().cpu().numpy()
    for of in (-1, 2, 3):
        c.r["allowed_of"] = np.full(6, of, np.int32)
        logits.check(ssd, c, k, want_adjust=False)
