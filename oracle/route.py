"""The router of a routed layer in float64: which branches a token takes, probabilities, counts, balance loss and gradient.

The loss is A * sum_b f_b P_b over the active branches: f_b the share of the assignments that go to branch b, P_b its mean
probability over the tokens that count.  The counts have no gradient.  A logit of minus infinity bars its branch; one that is
not a number is never taken, and its token counts, with probabilities that are not numbers.
"""
import numpy as np


def route_topk(logits, k, active=None, real=None):
    """(route [T, B] uint8, probs [T, B] float64, counts [B + 1] int64, loss)."""
    x = np.asarray(logits, dtype=np.float64)
    T, B = x.shape
    active = np.ones(B, bool) if active is None else np.asarray(active) != 0
    real = np.ones(T, bool) if real is None else np.asarray(real) != 0
    route = np.zeros((T, B), np.uint8)
    probs = np.zeros((T, B))
    counts = np.zeros(B + 1, np.int64)
    for t in range(T):
        on = [b for b in range(B) if active[b] and not x[t, b] == -np.inf]
        numbers = [b for b in on if not np.isnan(x[t, b])]
        if not real[t] or not on:
            continue
        counts[B] += 1
        top = max((x[t, b] for b in numbers), default=np.nan)
        with np.errstate(invalid="ignore"):
            e = {b: np.exp(x[t, b] - top) for b in on}
        s = sum(e.values())
        for b in on:
            probs[t, b] = e[b] / s
        for b in sorted(numbers, key=lambda b: (-x[t, b], b))[:k]:
            route[t, b] = 1
            counts[b] += 1
    taken = counts[:B].sum()
    loss = float(np.sum(0.0 * probs))                # 0, or not a number
    if taken:
        loss = float(active.sum()) * float(np.sum(counts[:B] / taken * probs.sum(axis=0))) / counts[B]
    return route, probs, counts, loss


def route_backward(probs, counts, dprobs=None, dloss=0.0, n_active=None):
    """Gradient of sum(dprobs * probs) + dloss * loss with respect to the logits, [T, B]."""
    p = np.asarray(probs, dtype=np.float64)
    T, B = p.shape
    A = B if n_active is None else n_active
    c = np.asarray(counts, dtype=np.float64)
    g = np.zeros((T, B)) if dprobs is None else np.array(dprobs, dtype=np.float64)
    if c[:B].sum() > 0:
        g = g + dloss * A * (c[:B] / c[:B].sum()) / c[B]
    g[p == 0] = 0.0
    return np.where(p == 0, 0.0, p * (g - (p * g).sum(axis=1, keepdims=True)))
