"""Filtered draws (temperature, top-k, top-p, min-p) in float64, one row at a time, entry by entry in the order that the
definition names: value descending, index ascending."""
import math

import numpy as np


def row_logits(logits, scale):
    """[R, V] float32 rows; scale > 0: the first half conditional, the second unconditional, float32 after every operation."""
    z = np.asarray(logits, dtype=np.float32)
    if scale > 0:
        R = z.shape[0] // 2
        d = (z[:R] - z[R:]).astype(np.float32)
        z = (z[R:] + (np.float32(scale) * d).astype(np.float32)).astype(np.float32)
    return np.where(np.isnan(z), np.float32(-np.inf), z)


def kept(z, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Weights of the entries that stay ({index: weight}) of one row of finite or -inf values."""
    z = np.asarray(z, dtype=np.float64)
    order = sorted((i for i in range(len(z)) if z[i] > -math.inf), key=lambda i: (-z[i], i))
    if not order:
        return {}
    if temperature == 0:
        return {order[0]: 1.0}
    top = z[order[0]]
    w = {i: (1.0 if z[i] == top else math.exp((z[i] - top) / temperature)) for i in order}
    if top_k:
        order = order[:top_k]
    if top_p < 1.0:
        limit, front, some = top_p * math.fsum(w[i] for i in order), [], 0.0
        for i in order:
            if some >= limit:
                break
            front.append(i)
            some += w[i]
        order = front
    return {i: w[i] for i in order if w[i] >= min_p}


def draw(weights, u):
    """First index whose inclusive mass exceeds u times all of it, and the distance of that threshold from the next border."""
    if not weights:
        return -1, math.inf
    at = sorted(weights)
    cum = np.cumsum([weights[i] for i in at])
    u = min(max(0.0 if u != u else float(u), 0.0), 1.0 - 2.0 ** -24)
    t = u * cum[-1]
    x = int(np.searchsorted(cum, t, side="right"))
    return at[min(x, len(at) - 1)], float(np.abs(cum - t).min() / cum[-1])
