"""Attention over a prefix that sequences share and the rows each has of its own, with a window and sinks: the
definition in float64, query by query, and the bounds its float32 and bf16 forms keep to."""
import math

import torch


def visible_keys(p, sinks, window):
    """Positions that the query at position p sees, in order."""
    return [t for t in range(p + 1) if window == 0 or t < sinks or p - t < window]


def context_attention(q, k, v, starts, pk=None, pv=None, S=0, sinks=0, window=0, scale=None):
    """q [B, nh, L, dh]; k [B, nkv, rows, dh]; v [B, nkv, dh, rows]; starts: own rows in front of each block (< 0: absent);
    pk [G, nkv, *, dh], pv [G, nkv, dh, *].  Returns out [B, nh, L, dh] float64 and, per query, what its rounding errors scale
    with: mass [B, nh, L, dh] = sum_t w_t |v_t| and reach [B, nh, L] = max_t scale sum_c |q_c k_tc|, keys [B, L]."""
    B, nh, L, dh = q.shape
    nkv = k.shape[1]
    scale = dh ** -0.5 if scale is None else scale
    q, k, v = q.double().cpu(), k.cpu(), v.cpu()
    out, mass = torch.zeros(B, nh, L, dh, dtype=torch.float64), torch.zeros(B, nh, L, dh, dtype=torch.float64)
    reach, keys = torch.zeros(B, nh, L, dtype=torch.float64), torch.zeros(B, L)
    for b in range(B):
        if starts[b] < 0:
            continue
        n = starts[b] + L
        K, Vt = k[b, :, :n].double(), v[b, :, :, :n].double()
        if S:
            g = b // (B // pk.shape[0])
            K = torch.cat([pk[g, :, :S].double().cpu(), K], 1)
            Vt = torch.cat([pv[g, :, :, :S].double().cpu(), Vt], 2)
        for j in range(L):
            at = visible_keys(S + starts[b] + j, sinks, window)
            keys[b, j] = len(at)
            Kj = K[:, at].repeat_interleave(nh // nkv, 0)                   # [nh, keys, dh]
            Vj = Vt[:, :, at].repeat_interleave(nh // nkv, 0)               # [nh, dh, keys]
            z = scale * (Kj @ q[b, :, j, :, None])[..., 0]
            e = torch.exp(z - z.max(-1, keepdim=True).values)
            w = e / e.sum(-1, keepdim=True)
            out[b, :, j] = (Vj @ w[..., None])[..., 0]
            mass[b, :, j] = (Vj.abs() @ w[..., None])[..., 0]
            reach[b, :, j] = (scale * (Kj.abs() @ q[b, :, j, :, None].abs())[..., 0]).max(-1).values
    return out, mass, reach, keys


def tolerance(mass, reach, keys, out, dh, bf16):
    """How far a form with float32 scores, statistics and sums may be off, by arithmetic.
    A score is a sum of dh products: off by at most dh 2^-24 reach, and as the argument of an exponential (times log2 e, less a
    reference) by 4 2^-24 of its size, which reach bounds twice; the exponential itself is good to 2^-22.  That moves every weight
    by the relative amount `d`, numerator and denominator together by 2 d.  The sums of n terms and the division add
    (n + 8) 2^-24, twice.  bf16: every weight in the numerator is rounded (half a step: 2^-8), and the output once more (2^-8 of it)."""
    d = (dh + 8) * 2.0 ** -24 * reach + 2.0 ** -22
    rel = 2 * d + 2 * (keys[:, None, :] + 8) * 2.0 ** -24
    tol = mass * rel[..., None]
    if bf16:
        tol = tol + 2.0 ** -8 * (mass + out.abs() + tol)
    else:
        tol = tol + 2.0 ** -24 * out.abs()
    return tol
