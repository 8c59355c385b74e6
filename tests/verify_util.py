"""Verification of drafted tokens in plain 64-bit numpy, from its definition: round by round, each with a row of its own."""
from __future__ import annotations

import numpy as np


def softmax(x, scale):
    """Probabilities of one row of logits; NaN has no weight, and +infinity shares all of it."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    if not scale > 0 or x.max() == -np.inf:
        return np.zeros(len(x))
    if x.max() == np.inf:
        e = (x == np.inf).astype(np.float64)
    else:
        e = np.exp(scale * (x - x.max()))
    return e / e.sum()


class Walk:
    """path, next and `sure`: the distance of the closest decision from its border, relative to what is compared."""

    def __init__(self):
        self.path, self.next, self.sure = [], -1, np.inf

    def closer(self, x, y, size):
        self.sure = min(self.sure, abs(x - y) / size if size > 0 else np.inf)


def draw(w, u, out):
    """The first entry whose running sum exceeds u times the whole."""
    run = np.cumsum(w)
    if len(w) == 0 or not run[-1] > 0:
        return -1
    mark = u * run[-1]
    t = int(np.searchsorted(run, mark, side="right"))
    t = min(t, int(np.nonzero(w)[0][-1]))
    for border in (run[t], run[t] - w[t]):
        if 0 < border < run[-1]:
            out.closer(mark, border, run[-1])
    return t


def walk(tokens, parent, live, target, draft, logits, scale, u):
    """One sequence.  target, draft: [n_draft, vocab] float64 rows; u None or scale infinite: greedy."""
    out, t, vocab = Walk(), len(target), target.shape[1]
    live = min(max(live, 0), t)
    if live == 0:
        return out
    node, out.path = 0, [0]
    greedy = u is None or (logits and scale == np.inf)
    probs = (lambda x: softmax(x, scale)) if logits else (lambda x: np.where(np.isnan(x), 0.0, x))
    while True:
        children = [j for j in range(node + 1, live) if parent[j] == node]
        if greedy:
            row = np.where(np.isnan(target[node]), -np.inf, target[node])
            out.next = int(np.argmax(row)) if row.max() > -np.inf else -1
            hit = next((j for j in children if tokens[j] == out.next and out.next >= 0), None)
            if hit is None:
                return out
        else:
            p = probs(target[node])
            q = probs(draft[node]) if draft is not None else None
            w, total, hit, refused = p, 1.0, None, set()
            for j in children:
                c = int(tokens[j])
                if not 0 <= c < vocab or c in refused:
                    continue
                if q is not None:  # against what the rounds before have left of p, as a distribution
                    left = w[c] / total if total > 0 else 0.0
                    out.closer(u[j] * q[c], left, max(u[j] * q[c], p[c]))
                    if u[j] * q[c] < left:
                        hit = j
                        break
                    w = np.maximum(w / total - q, 0.0) if total > 0 else w
                    total = w.sum()
                else:
                    out.closer(u[j] * total, p[c], max(total, p[c]))
                    if u[j] * total < p[c]:
                        hit = j
                        break
                    refused.add(c)
                    total -= p[c]
            if hit is None:
                if refused:
                    w = p.copy()
                    w[list(refused)] = 0.0
                elif not w.sum() > 0:
                    w = p
                out.next = draw(w, float(u[0]), out)
                return out
        node = hit
        out.path.append(node)
