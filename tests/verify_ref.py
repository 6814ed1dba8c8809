"""Draft verification in 64 bits, sequence by sequence (adept_verify_drafts' definition)."""
import math

import numpy as np


def law(logits, t):
    """The row's distribution at temperature t; None for a row without one."""
    x = np.where(np.isnan(logits), -np.inf, logits).astype(np.float64)
    top = x.max()
    if top == -np.inf:
        return None
    with np.errstate(over="ignore", invalid="ignore"):
        w = (x == np.inf).astype(float) if top == np.inf else np.exp((x - top) / t)
    return np.where(x == -np.inf, 0.0, w) / np.where(x == -np.inf, 0.0, w).sum()


def best(logits):
    x = np.where(np.isnan(logits), -np.inf, logits)
    return int(x.argmax()) if x.max() > -np.inf else -1


def draw(w, u):
    """The first index whose running sum exceeds u times the whole, else the last with a weight."""
    if w is None:
        return -1
    s = np.cumsum(w)
    over = np.nonzero((s > (u * s[-1] if u > 0 else 0.0)) & (w > 0))[0]
    return int(over[0] if len(over) else np.nonzero(w)[0][-1])


def verify(target, draft, tokens, u, n_draft=None, temperature=None):
    target = np.asarray(target, np.float64)
    n, rows, V = target.shape
    out, kept = np.full((n, rows), -1, np.int32), np.zeros(n, np.int32)
    for b in range(n):
        g = rows - 1 if n_draft is None else min(max(int(n_draft[b]), 0), rows - 1)
        t = 1.0 if temperature is None else float(temperature[b])
        greedy = not t > 0
        rest, i = None, 0
        while i < g:
            x = int(tokens[b][i])
            there = 0 <= x < V
            if greedy:
                if not there or best(target[b, i]) != x:
                    break
            else:
                p = law(target[b, i], t)
                if draft is None:
                    q, qx = np.zeros(V), 1.0
                    if there:
                        q[x] = math.inf
                else:
                    q = law(np.asarray(draft[b, i], np.float64), t)
                    q = np.zeros(V) if q is None else q
                    qx = q[x] if there else 0.0
                px = p[x] if there and p is not None else 0.0
                if not float(u[b][i]) * qx < px:
                    rest = None if p is None else np.maximum(p - q, 0)
                    break
            out[b, i] = x
            i += 1
        kept[b] = i
        if greedy:
            out[b, i] = best(target[b, i])
            continue
        if rest is None or rest.sum() == 0:
            rest = law(target[b, i], t)
        out[b, i] = draw(rest, float(u[b][rows - 1]))
    return out, kept
