"""The operators of ssd_ops.h in plain numpy, 64 bits, request by request."""
import math

import numpy as np


def plan(row_start, lens, parents, table, held, ring, ends, page, n_pages, n_rows, words, bad=-7):
    """Returns a dict of the outputs; table and ring are copies with the call's changes.  Rows that no request owns hold `bad`."""
    table, ring = table.copy(), ring.copy()
    B, width = table.shape
    head, tail = int(ends[0]), int(ends[1])
    slots, positions = np.full(n_rows, bad, np.int32), np.full(n_rows, bad, np.int32)
    masks = np.full((n_rows, words), bad, np.int64).view(np.uint64) if words else None
    held_out, status = held.copy(), 0
    short, at, pops, pushes = False, head, 0, []
    for b in range(B):
        rows = range(row_start[b], row_start[b + 1])
        given = False
        if lens[b] < 0:
            pushes += table[b, :held[b]].tolist()
            held_out[b] = 0
        else:
            need = -(-(int(lens[b]) + len(rows)) // page)
            fresh = max(0, need - int(held[b]))
            if need > width:
                status |= 2
            elif fresh == 0:
                given = True
            elif short or pops + fresh > tail - head:
                short = True
                status |= 1
            else:
                given = True
                for j in range(int(held[b]), need):
                    table[b, j] = ring[at % n_pages]
                    at += 1
                pops += fresh
                held_out[b] = need
        depth, seen = [], []
        for i, r in enumerate(rows):
            x = int(lens[b]) + i
            if given:
                slots[r] = table[b, x // page] * page + x % page
            else:
                slots[r] = -1
            if parents is None:
                positions[r] = x
                continue
            p = int(parents[r])
            if i >= 64 * words:
                status |= 4
                depth.append(0)
                seen.append(0)
            else:
                if p < -1 or p >= i:
                    status |= 4
                    p = -1
                depth.append(depth[p] + 1 if p >= 0 else 0)
                seen.append((1 << i) | (seen[p] if p >= 0 else 0))
            positions[r] = int(lens[b]) + depth[i]
            for k in range(words):
                masks[r, k] = (seen[i] >> (64 * k)) & (2**64 - 1)
    for i, p in enumerate(pushes):
        ring[(tail + i) % n_pages] = p
    return {"table": table, "ring": ring, "held": held_out, "ends": np.array([head + pops, tail + len(pushes)]), "slots": slots,
            "positions": positions, "masks": None if masks is None else masks.view(np.int64), "status": status}


def frequencies(rot, theta=1e4, scaling=0, factor=1.0, original=0.0, slow=1.0, fast=32.0):
    f = theta ** (-2.0 * np.arange(rot // 2) / rot)
    if scaling == 1:
        return f / factor
    if scaling == 2:
        g = np.clip((original * f / (2 * math.pi) - slow) / (fast - slow), 0, 1)
        return f * (g + (1 - g) / factor)
    return f


def rope(x, positions, f, interleaved, amplitude=1.0):
    """x [n][heads][hd] turned, in float64."""
    x = np.asarray(x, np.float64).copy()
    a = np.asarray(positions, np.float64)[:, None] * f[None]
    c, s = (amplitude * np.cos(a))[:, None], (amplitude * np.sin(a))[:, None]
    n = len(f)
    lo, hi = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    u, w = x[..., lo].copy(), x[..., hi].copy()
    x[..., lo], x[..., hi] = u * c - w * s, w * c + u * s
    return x


def gather(cache, table_row, total, page, n_pages):
    """Rows 0 .. total-1 of a request [total][kv_head][dim] from one layer [page][kv_head][pos][dim]; pages outside: zeros."""
    x = np.arange(total)
    p = table_row[x // page]
    ok = (p >= 0) & (p < n_pages)
    out = cache[np.where(ok, p, 0), :, x % page].astype(np.float64)
    out[~ok] = 0
    return out


def attention(q, k, v, row_start, lens, table, page, masks, scale):
    """q [n][H][hd]; k, v [page][kv_head][pos][dim].  Returns (out float64, rows written, bounds): per row and head, the
    largest |v| it sees, the largest scale * sum |q k| and the number of positions."""
    n, H, hd = q.shape
    Hkv, G = k.shape[1], H // k.shape[1]
    out = np.zeros((n, H, hd))
    vmax, smax, count = np.zeros((n, H)), np.zeros((n, H)), np.zeros((n, 1))
    written = np.zeros(n, bool)
    for b in range(len(lens)):
        r0, r1 = row_start[b], row_start[b + 1]
        if lens[b] < 0 or r1 == r0:
            continue
        total = min(int(lens[b]) + r1 - r0, table.shape[1] * page)
        kk, vv = (gather(c, table[b], total, page, k.shape[0]) for c in (k, v))
        for r in range(r0, r1):
            written[r] = True
            j = np.arange(total) - int(lens[b])
            if masks is None:
                seen = j <= r - r0
            else:
                m = masks[r].view(np.uint64)
                jj = np.clip(j, 0, 64 * len(m) - 1)
                seen = (j < 0) | ((j < 64 * len(m)) & ((m[jj // 64] >> (jj % 64).astype(np.uint64)) & np.uint64(1) == 1))
            at = np.nonzero(seen)[0]
            count[r] = len(at)
            for h in range(H):
                g = h // G
                if not len(at):
                    continue
                prod = kk[at, g] * q[r, h].astype(np.float64)
                s = scale * prod.sum(1)
                top = s.max()
                if top == -np.inf:
                    continue
                with np.errstate(invalid="ignore"):
                    w = np.exp(s - top)
                    out[r, h] = (w[:, None] * vv[at, g]).sum(0) / w.sum()
                vmax[r, h] = np.abs(vv[at, g]).max()
                smax[r, h] = scale * np.abs(prod).sum(1).max()
    return out, written, (vmax, smax, count)


def commit(row_start, lens, table, page, parents, tokens, target, n_rows, bad=-7):
    """Outputs and the moves [(request, from index, to index)] in order."""
    B = len(lens)
    acc, nxt, new = np.full(B, -1, np.int32), np.full(B, -1, np.int32), np.array(lens, np.int32)
    path, emitted = np.full(n_rows, bad, np.int32), np.full(n_rows, bad, np.int32)
    moves = []
    for b in range(B):
        r0 = row_start[b]
        n = min(row_start[b + 1] - r0, 256)
        if n == 0 or lens[b] < 0:
            continue
        at, steps = 0, [0]
        while True:
            below = [i for i in range(at + 1, n) if (i - 1 if parents is None else parents[r0 + i]) == at and tokens[r0 + i] == target[r0 + at]]
            if not below:
                break
            at = below[0]
            steps.append(at)
        acc[b], nxt[b], new[b] = len(steps) - 1, target[r0 + at], lens[b] + len(steps)
        for j, s in enumerate(steps):
            path[r0 + j] = s
            emitted[r0 + j] = tokens[r0 + steps[j + 1]] if j + 1 < len(steps) else target[r0 + at]
            if s != j:
                moves.append((b, lens[b] + s, lens[b] + j))
    return acc, nxt, new, path, emitted, moves
