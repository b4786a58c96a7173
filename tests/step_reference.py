"""The operators of ssd_step.h in plain numpy, 64 bits, row by row."""
import math

import numpy as np


def axis_of_pair(half, n_axes, pairs, in_turns):
    if not in_turns:
        return [a for a in range(n_axes) for _ in range(pairs[a])]
    left, out = list(pairs), []
    for i in range(half):
        a = i % n_axes
        if i // n_axes < left[a]:
            out.append(a)
        else:
            out.append(0)
    return out


def turned(x, gain, eps, positions, axis, rates, rot, interleaved, amplitude=1.0):
    """x [head][hd] of one row, positions [axis]: normalised, then the first rot dims turned."""
    x = x.astype(np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain.astype(np.float64)
    y = x.copy()
    for i in range(rot // 2):
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        t = float(positions[axis[i]]) * rates[i]
        c, s = amplitude * math.cos(t), amplitude * math.sin(t)
        y[:, lo], y[:, hi] = x[:, lo] * c - x[:, hi] * s, x[:, hi] * c + x[:, lo] * s
    return y


def adjusted(logits, vocab, b, row, node, start, count, r):
    """One row's logits after the rules r (a dict of numpy arrays as LogitRules takes them), every step rounded to fp32 as the
    operator does.  b: its request, node: its index there, start: the request's first row, count: the request's rows."""
    x = logits.astype(np.float32).copy()
    f32 = np.float32
    own, prompt = np.zeros(vocab, np.int64), np.zeros(vocab, bool)
    if any(r.get(p) is not None for p in ("repetition", "presence", "frequency")):
        if r.get("history") is not None:
            n = min(max(int(r["history_len"][b]), 0), r["history"].shape[1])
            before = int(r["prompt_len"][b]) if r.get("prompt_len") is not None else 0
            for j in range(n):
                t = int(r["history"][b, j])
                if 0 <= t < vocab:
                    if j < before:
                        prompt[t] = True
                    else:
                        own[t] += 1
        if r.get("tokens") is not None:
            for j in range(count):
                if r.get("masks") is None:
                    seen = j <= node
                else:
                    seen = j < 64 * r["masks"].shape[1] and (int(r["masks"][row, j // 64]) >> (j % 64)) & 1
                t = int(r["tokens"][start + j])
                if seen and 0 <= t < vocab:
                    own[t] += 1
        with np.errstate(all="ignore"):
            said = prompt | (own > 0)
            p = f32(r["repetition"][b]) if r.get("repetition") is not None else f32(1)
            x = np.where(said, np.where(x > 0, x / p, x * p), x).astype(f32)
            if r.get("frequency") is not None:
                x = np.where(said, x - f32(r["frequency"][b]) * own.astype(f32), x).astype(f32)
            if r.get("presence") is not None:
                x = np.where(own > 0, x - f32(r["presence"][b]), x).astype(f32)
    if r.get("bias") is not None:
        i = int(r["bias_of"][b]) if r.get("bias_of") is not None else 0
        if 0 <= i < r["bias"].shape[0]:
            x = (x + r["bias"][i]).astype(f32)
    if r.get("allowed") is not None:
        i = int(r["allowed_of"][row]) if r.get("allowed_of") is not None else row
        if 0 <= i < r["allowed"].shape[0]:
            t = np.arange(vocab)
            ok = (r["allowed"][i].view(np.uint32)[t // 32] >> (t % 32).astype(np.uint32)) & 1
            x = np.where(ok == 1, x, f32(-np.inf))
    return x


def chosen(x, k):
    """(tokens, log probabilities, logsumexp) of the k best of one row."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    order = np.argsort(-x, kind="stable")[:k]
    order = [int(i) for i in order if x[i] > -np.inf]
    if not order:
        return [-1] * k, [-np.inf] * k, -np.inf
    top = x[order[0]]
    if top == np.inf:
        n = math.log(int((x == np.inf).sum()))
        lp, total = [-n if x[i] == np.inf else -np.inf for i in order], np.inf
    else:
        total = top + math.log(np.exp(x - top).sum())
        lp = [x[i] - total for i in order]
    pad = k - len(order)
    return order + [-1] * pad, lp + [-np.inf] * pad, total


def routed(x, w, k, favour, sigmoid, renorm, scale):
    """(ids, weights) of rows x."""
    z = x.astype(np.float64) @ w.astype(np.float64).T
    if sigmoid:
        p = 1.0 / (1.0 + np.exp(-z))
    else:
        p = np.exp(z - z.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
    score = p if favour is None else p + favour.astype(np.float64)
    ids = np.argsort(-score, axis=-1, kind="stable")[:, :k]
    q = np.take_along_axis(p, ids, -1)
    if renorm:
        q = q / q.sum(-1, keepdims=True)
    return ids, q * scale


def mlp(x, ids, weights, gate, up, down, residual, step):
    """(result, bound of the error in front of the last rounding) of rows x.  step: half a step of the type.

    A product of n values is summed in at most n / 16 + 20 additions, each off by at most 2^-22 of the terms' absolute sum (the matrix
    instructions cut off instead of rounding); silu has a slope of at most 1.1; h enters as a pair, off by step^2."""
    out = np.zeros(x.shape) if residual is None else residual.astype(np.float64).copy()
    err = 2.0**-22 * np.abs(out)
    c = [(n / 16 + 20) * 2.0**-22 for n in (gate.shape[2], down.shape[2])]
    for r in range(x.shape[0]):
        for j in range(ids.shape[1]):
            e = int(ids[r, j])
            if not 0 <= e < gate.shape[0]:
                continue
            v, g, q, m = (t.astype(np.float64) for t in (x[r], gate[e], up[e], down[e]))
            a, u = g @ v, q @ v
            s = a / (1.0 + np.exp(-a))
            h = s * u
            dh = 1.1 * c[0] * (np.abs(g) @ np.abs(v)) * np.abs(u) + np.abs(s) * c[0] * (np.abs(q) @ np.abs(v)) + np.abs(h) * (step * step + 2.0**-21) + 2.0**-25 * (step < 2.0**-9)
            w = float(weights[r, j])
            out[r] += w * (m @ h)
            err[r] += abs(w) * (np.abs(m) @ (dh + c[1] * np.abs(h))) + ids.shape[1] * 2.0**-23 * abs(w) * np.abs(m @ h)
    return out, err
