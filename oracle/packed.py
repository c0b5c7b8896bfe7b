"""A cache in 4 or 8 bits: the numbers its codes stand for, which codes a row gets, where they lie, and attention over
them, in float64.  Formats are "fp4" and "fp8"."""
import numpy as np
import torch

from . import context as OC

TILE, GROUP = 64, 32
# bits, exponent bits and bias, mantissa bits, codes that are numbers (without the sign), what a group may reach, largest group exponent
FORMATS = {"fp4": dict(bits=4, mant=1, bias=1, codes=8, reach=7.0, cap=125), "fp8": dict(bits=8, mant=3, bias=7, codes=127, reach=464.0, cap=119)}


def grid(fmt):
    """The numbers of the format that are not negative, by code."""
    f = FORMATS[fmt]
    out = []
    for code in range(f["codes"]):
        e, m = divmod(code, 1 << f["mant"])
        m /= 1 << f["mant"]
        out.append(m * 2.0 ** (1 - f["bias"]) if e == 0 else (1 + m) * 2.0 ** (e - f["bias"]))
    return np.array(out)


def encode(x, fmt):
    """Codes and scale bytes of rows x [.., dh]: the smallest exponent whose grid reaches the group's largest number, then for every number
    the nearer of the two neighbours on the grid (halfway: the even code)."""
    f, G = FORMATS[fmt], grid(fmt)
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    m = np.abs(g).max(-1)
    bad = ~np.isfinite(m)
    m = np.where(bad, 0.0, m)
    exps = np.arange(-117, f["cap"] + 1)
    e = exps[np.minimum(np.searchsorted(f["reach"] * 2.0 ** exps, m), len(exps) - 1)]
    y = np.abs(np.where(bad[..., None], 0.0, g)) / 2.0 ** e[..., None]
    hi = np.clip(np.searchsorted(G, y), 1, len(G) - 1)
    lo = hi - 1
    to_lo, to_hi = y - G[lo], G[hi] - y
    code = np.where(to_lo < to_hi, lo, np.where(to_hi < to_lo, hi, np.where(lo % 2 == 0, lo, hi)))
    code = code + np.signbit(g) * (1 << (f["bits"] - 1))
    code = np.where(bad[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def decode(code, scale, fmt):
    f, G = FORMATS[fmt], grid(fmt)
    G = np.concatenate([G, np.full((1 << (f["bits"] - 1)) - len(G), np.nan)])
    G = np.concatenate([G, -G])
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return G[code] * np.repeat(s, GROUP, -1)


def tile_bytes(fmt, dh):
    return TILE * dh * FORMATS[fmt]["bits"] // 8 + TILE * dh // GROUP


def places(fmt, dh, keys):
    """For a tile: index of the code of (row, channel), and byte of the scale of (row, group)."""
    r, c = np.arange(TILE)[:, None], np.arange(dh)[None, :]
    g, G, u = np.arange(dh // GROUP)[None, :], dh // GROUP, dh // 16
    first = TILE * dh * FORMATS[fmt]["bits"] // 8
    if keys:
        return r * dh + c, first + ((r % 16) * G + g) * 4 + r // 16
    return (r // 4) * 4 * dh + (c // u) * 4 * u + (r % 4) * u + c % u, first + ((r // 4 % 4 * G + g) * 4 + r // 16) * 4 + r % 4


def to_tiles(code, scale, fmt, keys):
    """Tiles [.., rows / 64, tile bytes] of codes [.., rows, dh] and scale bytes [.., rows, dh / 32]."""
    *lead, rows, dh = code.shape
    at, scale_at = places(fmt, dh, keys)
    code = code.reshape(*lead, rows // TILE, TILE, dh)
    scale = scale.reshape(*lead, rows // TILE, TILE, dh // GROUP)
    flat = np.zeros((*lead, rows // TILE, TILE * dh), np.uint8)
    flat[..., at] = code
    out = np.zeros((*lead, rows // TILE, tile_bytes(fmt, dh)), np.uint8)
    n = TILE * dh * FORMATS[fmt]["bits"] // 8
    out[..., :n] = flat if fmt == "fp8" else flat[..., ::2] | flat[..., 1::2] << 4
    out[..., scale_at] = scale
    return out


def from_tiles(tiles, fmt, dh, keys):
    """Codes and scale bytes, the other way round."""
    at, scale_at = places(fmt, dh, keys)
    n = TILE * dh * FORMATS[fmt]["bits"] // 8
    flat = tiles[..., :n]
    if fmt == "fp4":
        flat = np.stack([flat & 15, flat >> 4], -1).reshape(*flat.shape[:-1], 2 * n)
    lead = tiles.shape[:-2]
    return flat[..., at].reshape(*lead, -1, dh), tiles[..., scale_at].reshape(*lead, -1, dh // GROUP)


def packed_attention(q, k, v, starts, sinks=0, window=0, scale=None):
    """context_attention over numbers k, v [B, nkv, rows, dh] of the cache.  Besides its results: group_reach [B, nh, L] =
    max_t scale sum_c (largest |q| of the group of c) |k_tc|, over the rows a query sees."""
    B, nh, L, dh = q.shape
    out, mass, reach, keys = OC.context_attention(q, k, v.transpose(2, 3), starts, sinks=sinks, window=window, scale=scale)
    return out, mass, reach, keys, group_reach(q, k, starts, sinks, window, scale)


def group_reach(q, k, starts, sinks=0, window=0, scale=None):
    B, nh, L, dh = q.shape
    scale = dh ** -0.5 if scale is None else scale
    most = q.double().abs().cpu().unflatten(-1, (-1, GROUP)).amax(-1, keepdim=True).expand(-1, -1, -1, -1, GROUP).flatten(-2)
    found = torch.zeros(B, nh, L, dtype=torch.float64)
    for b in range(B):
        for j in range(L if starts[b] >= 0 else 0):
            at = OC.visible_keys(starts[b] + j, sinks, window)
            kj = k[b, :, at].double().abs().repeat_interleave(nh // k.shape[1], 0)
            found[b, :, j] = (scale * (kj @ most[b, :, j, :, None])[..., 0]).max(-1).values
    return found


def tolerance(mass, reach, keys, out, dh, bf16, grouped, largest):
    """How far a form with float32 sums may be off.  Numbers of the cache are exact in bf16; a bf16 query enters the scores as two terms of four
    significant bits each, which hold it but for 2^-21 of the largest of its group of 32, a float32 query as three bf16 terms, which hold it but
    for 2^-24: a score is a sum of 2 dh or 3 dh products, off by (3 dh + 8) 2^-24 reach and (bf16) 2^-21 grouped.  As the argument of
    an exponential it is off by 4 2^-24 of its size twice more, which the 8 counts; the exponential is good to 2^-22.  Every weight
    then by the relative amount d, numerator and denominator together by 2 d.  float32 exponentials enter the second product as
    three bf16 terms (2^-24, and 3 n terms to add).  Sums of n terms and the division: (3 n + 8) 2^-24, twice.  bf16: half a step of 2^-8 of
    every weight, and of the output.  What lies below 2^-126, float32's and bf16's smallest number of full precision, may count as 0: an
    exponential (relative to the largest, which is at least 2^-8), its three terms, its product with a value, a partial result and the
    output.  `largest` is the largest |v|: n exponentials lose up to n 2^-116 of it, and four roundings of sums 2^-124."""
    d = (3 * dh + 8) * 2.0 ** -24 * reach + 2.0 ** -22 + (2.0 ** -21 * grouped if bf16 else 2.0 ** -24)
    rel = 2 * d + 2 * (3 * keys[:, None, :] + 8) * 2.0 ** -24
    tol = mass * rel[..., None] + 2.0 ** -116 * keys[:, None, :, None] * largest + 2.0 ** -124
    return tol + 2.0 ** -8 * (mass + out.abs() + tol) if bf16 else tol + 2.0 ** -24 * out.abs()
