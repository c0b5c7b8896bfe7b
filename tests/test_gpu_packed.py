"""mulo_pack_rows, mulo_unpack_rows and mulo_packed_attention through the C ABI against their definitions (oracle/packed.py): every byte of a
cache, and attention over formats, types, head layouts, lengths, windows, ragged and absent sequences, strides and memory that
nothing may read."""
import numpy as np
import pytest
import torch

import paper_2601_05149_amd as mulo
from oracle import packed as OP
from tests.gpu_util import DEV, say

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
FMT = {"fp4": mulo.MULO_FP4, "fp8": mulo.MULO_FP8}
NAN = float("nan")


# ---- rows in, rows out ----------------------------------------------------------------------------------------------
def packed_of(tiles_k, tiles_v, fmt, dh):
    return mulo.make_packed_kv(tiles_k, tiles_v, FMT[fmt], dh)


def layout(t, how):
    """The numbers t [B, nkv, L, dh] in another order in memory, same indexes."""
    if how == "rows":
        return t.contiguous()
    if how == "tokens":          # a token's heads next to each other
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    if how == "wide":            # inside wider rows, heads in front of sequences
        B, n, L, dh = t.shape
        w = torch.full((n, B, L, 2 * dh), NAN, dtype=t.dtype, device=t.device)
        w[..., dh:] = t.transpose(0, 1)
        return w[..., dh:].transpose(0, 1)
    if how == "channels":        # channels of rows
        return t.transpose(2, 3).contiguous().transpose(2, 3)
    B, n, L, dh = t.shape        # channels of rows inside longer ones, from an odd place on
    w = torch.full((B, n, dh, L + 13), NAN, dtype=t.dtype, device=t.device)
    w[..., 5:5 + L] = t.transpose(2, 3)
    return w[..., 5:5 + L].transpose(2, 3)


def numbers(B, nkv, L, dh, dtype, seed):
    """Groups of very different sizes, zeros, halfway numbers, a few that are none."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(B, nkv, L, dh)) * np.repeat(2.0 ** rng.integers(-20, 20, (B, nkv, L, dh // 32)), 32, -1)
    x[rng.random(x.shape) < 0.02] = 0
    at = rng.random((B, nkv, L)) < 0.2
    x[at, :32] = np.tile([0.25, -0.75, 1.25, -1.75, 2.5, -3.5, 5, 6], 4) * 2.0 ** rng.integers(-40, 40, (at.sum(), 1))
    at = rng.random((B, nkv, L)) < 0.05
    x[at, 32:64] = 0
    x[rng.random(x.shape) < 2e-4] = np.nan
    x[rng.random(x.shape) < 2e-4] = -np.inf
    return torch.tensor(x).to(DT[dtype])


def expected(before, x, starts, fmt, keys):
    """The cache's bytes after rows x [B, nkv, L, dh] have been written from starts[b] on."""
    dh = x.shape[-1]
    code, scale = OP.from_tiles(before, fmt, dh, keys)
    c, s = OP.encode(x.double().numpy(), fmt)
    for b, p in enumerate(starts):
        if p >= 0:
            code[b, :, p:p + x.shape[2]], scale[b, :, p:p + x.shape[2]] = c[b], s[b]
    return OP.to_tiles(code, scale, fmt, keys)


ROWS = [
    # format, type, dh, B, nkv, L, rows, P, starts, layout of k, of v
    ("fp4", "bf16", 128, 1, 1, 1, 64, 0, None, "rows", "rows"),
    ("fp4", "bf16", 128, 3, 2, 1, 128, 63, None, "tokens", "tokens"),
    ("fp4", "bf16", 64, 5, 3, 1, 192, 190, [0, 63, 64, -1, 1000], "tokens", "channels"),
    ("fp8", "bf16", 128, 2, 3, 7, 128, 60, None, "rows", "odd"),
    ("fp8", "bf16", 64, 2, 2, 130, 256, 61, [61, 3], "wide", "wide"),
    ("fp4", "f32", 128, 2, 2, 65, 192, 127, [127, 0], "tokens", "odd"),
    ("fp8", "f32", 64, 3, 2, 33, 128, 95, [95, -5, 30], "wide", "channels"),
    ("fp4", "bf16", 128, 2, 4, 300, 320, 17, None, "rows", "channels"),
    ("fp8", "f32", 128, 1, 2, 129, 192, 63, None, "rows", "rows"),
    ("fp4", "f32", 64, 2, 1, 64, 64, 0, None, "rows", "odd"),
    ("fp4", "bf16", 64, 70, 9, 3, 64, 61, None, "tokens", "rows"),
    ("fp8", "bf16", 128, 33, 7, 1, 64, 5, None, "tokens", "channels"),
]


def garbage(shape, seed):
    return np.random.default_rng(seed).integers(0, 256, shape, dtype=np.uint8)


@pytest.mark.parametrize("case", ROWS, ids=lambda c: "%s-%s-%d-%dx%d-L%d-P%d-%s-%s" % (c[:6] + (c[7],) + c[9:]))
def test_rows_in_and_out(case):
    fmt, dtype, dh, B, nkv, L, rows, P, starts, how_k, how_v = case
    shape = (B, nkv, rows // 64, OP.tile_bytes(fmt, dh))
    before = [garbage(shape, 1), garbage(shape, 2)]
    tiles = [torch.tensor(t, device=DEV) for t in before]
    x = [numbers(B, nkv, L, dh, dtype, 3), numbers(B, nkv, L, dh, dtype, 4)]
    k, v = layout(x[0].to(DEV), how_k), layout(x[1].to(DEV), how_v)
    P_seq = None if starts is None else torch.tensor(starts, dtype=torch.int32, device=DEV)
    packed, where = packed_of(*tiles, fmt, dh), [min(p, rows - L) for p in starts or [P] * B]
    mulo.mulo_pack_rows(packed, mulo.make_kv_rows(k, v, P, P_seq))
    torch.cuda.synchronize()
    for t, b, y, keys in zip(tiles, before, x, (True, False)):
        want = expected(b, y, where, fmt, keys)
        assert np.array_equal(t.cpu().numpy(), want), "%s: %d bytes differ" % ("keys" if keys else "values", (t.cpu().numpy() != want).sum())
    # and back, into memory that holds something
    outs = []
    for y, how in zip(x, (how_k, how_v)):
        outs.append(layout(torch.full_like(y, 7.0, device=DEV), how))
    mulo.mulo_unpack_rows(packed, mulo.make_kv_rows(*outs, P, P_seq))
    torch.cuda.synchronize()
    for o, t, keys in zip(outs, tiles, (True, False)):
        y = OP.decode(*OP.from_tiles(t.cpu().numpy(), fmt, dh, keys), fmt)
        for b, p in enumerate(where):
            want = torch.full((nkv, L, dh), 7.0) if p < 0 else torch.tensor(y[b, :, p:p + L]).float()
            got = o[b].float().cpu()
            assert torch.equal(torch.nan_to_num(got, nan=12345.0), torch.nan_to_num(want, nan=12345.0))
            assert torch.equal(torch.signbit(got) & ~got.isnan(), torch.signbit(want) & ~want.isnan())
        if o.untyped_storage().nbytes() > o.numel() * o.element_size():      # what lies between the rows
            assert torch.isnan(torch.as_strided(o, (o.storage_offset(),), (1,), 0).float()).all()


def inside(shape, how, dtype, device):
    """A buffer of sevens and a view [B, nkv, L, dh] into it that has some of them on every side: rows of channels, or channels of rows, from a
    place of 16 bytes on and whole pieces of them apart, or from an odd place on."""
    B, n, L, dh = shape
    if how == "rows":
        w = torch.full((n, B, L + 2, 3 * dh), 7.0, dtype=dtype, device=device)
        return w, w[:, :, 1:1 + L, dh:2 * dh].transpose(0, 1)
    first, wide = (8, (L + 23) // 8 * 8) if how == "whole" else (5, L + 13)
    w = torch.full((B, n, dh + 2, wide), 7.0, dtype=dtype, device=device)
    return w, w[:, :, 1:1 + dh, first:first + L].transpose(2, 3)


def outside_is_seven(w, view):
    own = torch.zeros(w.numel(), dtype=torch.bool, device=w.device)
    own.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(True)
    return bool((w.flatten()[~own] == 7).all())


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype, dh", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("how", ["rows", "whole", "odd"])
def test_nothing_around_the_rows_is_written(fmt, dtype, dh, how):
    """Rows read back into the middle of a buffer, at lengths that end inside a piece of 16 bytes, inside a tile and behind one; one of the
    sequences is absent."""
    B, nkv, rows = 3, 2, 320
    for L in (1, 2, 3, 7, 8, 9, 33, 63, 64, 65, 71, 127, 130):
        x = [numbers(B, nkv, L, dh, dtype, i) for i in (1, 2)]
        packed = mulo.alloc_packed_kv(B, nkv, rows, dh, FMT[fmt], DEV)
        starts = torch.tensor([rows - L, -1, 61], dtype=torch.int32, device=DEV)
        mulo.mulo_pack_rows(packed, mulo.make_kv_rows(*(t.to(DEV) for t in x), rows - L, starts))
        (wk, k), (wv, v) = inside(x[0].shape, "rows", DT[dtype], DEV), inside(x[1].shape, how, DT[dtype], DEV)
        mulo.mulo_unpack_rows(packed, mulo.make_kv_rows(k, v, rows - L, starts))
        torch.cuda.synchronize()
        for t, w, out in zip(x, (wk, wv), (k, v)):
            assert outside_is_seven(w, out) and (out[1] == 7).all(), L
            want = torch.tensor(OP.decode(*OP.encode(t.double().numpy(), fmt), fmt))
            assert torch.equal(torch.nan_to_num(out[::2].double().cpu(), nan=5.5), torch.nan_to_num(want[::2], nan=5.5)), L


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_keys_or_values_alone(fmt):
    x = numbers(2, 2, 5, 64, "bf16", 9)
    for alone in (0, 1):
        before = [garbage((2, 2, 1, OP.tile_bytes(fmt, 64)), i) for i in (1, 2)]
        tiles = [torch.tensor(t, device=DEV) for t in before]
        rows = [None, None]
        rows[alone] = x.to(DEV)
        mulo.mulo_pack_rows(packed_of(*tiles, fmt, 64), mulo.make_kv_rows(*rows, 20))
        out = [None, None]
        out[alone] = torch.empty_like(rows[alone])
        mulo.mulo_unpack_rows(packed_of(*tiles, fmt, 64), mulo.make_kv_rows(*out, 20))
        torch.cuda.synchronize()
        assert np.array_equal(tiles[alone].cpu().numpy(), expected(before[alone], x, [20, 20], fmt, alone == 0))
        assert np.array_equal(tiles[1 - alone].cpu().numpy(), before[1 - alone])
        want = OP.decode(*OP.encode(x.double().numpy(), fmt), fmt)
        assert torch.equal(torch.nan_to_num(out[alone].double().cpu(), nan=5.5), torch.nan_to_num(torch.tensor(want), nan=5.5))


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_number_of_a_group(fmt, dtype):
    """All bf16 numbers beside a largest one of several sizes (the least and the greatest exponents of a group among them); float32:
    the neighbours of every halfway number too."""
    top = float(OP.grid(fmt)[-1])
    rows = []
    for e in (-126, -117, -116, -40, 0, 3, 60, OP.FORMATS[fmt]["cap"] - 1, OP.FORMATS[fmt]["cap"]):
        most = top * 2.0 ** e
        if dtype == "bf16":
            v = (torch.arange(65536, dtype=torch.int32) << 16).view(torch.float32)
        else:
            G = torch.tensor(OP.grid(fmt))
            mid = ((G[1:] + G[:-1]) / 2 * 2.0 ** e).float()
            near = torch.stack([mid, torch.nextafter(mid, torch.tensor(0.0)), torch.nextafter(mid, torch.tensor(torch.inf))]).flatten()
            v = torch.cat([near, -near, (torch.rand(20000, generator=torch.Generator().manual_seed(1)) * 2 - 1) * most])
        v = v[v.isfinite() & (v.double().abs() <= most)]
        v = torch.cat([v, v.new_zeros(-len(v) % 31)]).reshape(-1, 31)
        rows.append(torch.cat([v.new_full((len(v), 1), most), v], 1))
    # numbers beyond what the largest exponent reaches
    big = torch.tensor([3.38e38, -3.38e38, 2.6e38, 3e38, 1.7e38, -2e38, 1.0, 0.0]).repeat(4)[None]
    x = torch.cat(rows + [big]).to(DT[dtype])
    x = torch.cat([x, x.new_zeros(-len(x) % 2, 32)]).reshape(1, 1, -1, 64)
    L = x.shape[2]
    tiles = [torch.zeros(1, 1, (L + 63) // 64, OP.tile_bytes(fmt, 64), dtype=torch.uint8, device=DEV) for _ in range(2)]
    before = [t.cpu().numpy() for t in tiles]
    mulo.mulo_pack_rows(packed_of(*tiles, fmt, 64), mulo.make_kv_rows(x.to(DEV), x.to(DEV), 0))
    torch.cuda.synchronize()
    for t, b, keys in zip(tiles, before, (True, False)):
        want_c, want_s = OP.from_tiles(expected(b, x, [0], fmt, keys), fmt, 64, keys)
        c, s = OP.from_tiles(t.cpu().numpy(), fmt, 64, keys)
        bad = np.argwhere(c[0, 0, :L] != want_c[0, 0, :L])
        assert np.array_equal(s, want_s) and not len(bad), "%d differ, first %s: %s" % (len(bad), bad[:1], x[0, 0, bad[0][0], bad[0][1]] if len(bad) else "")


def test_rows_beyond_32_bits():
    """The last rows of a cache longer than 2^32 bytes, and a head behind them."""
    rows, dh = 1 << 24, 128
    tiles = [torch.empty(1, 3, rows // 64, OP.tile_bytes("fp8", dh), dtype=torch.uint8, device=DEV) for _ in range(2)]
    x = numbers(1, 3, 70, dh, "bf16", 5)
    rows_in = mulo.make_kv_rows(x.to(DEV), x.to(DEV), rows - 70)
    packed = packed_of(*tiles, "fp8", dh)
    mulo.mulo_pack_rows(packed, rows_in)
    out = [torch.empty_like(x, device=DEV) for _ in range(2)]
    mulo.mulo_unpack_rows(packed, mulo.make_kv_rows(*out, rows - 70))
    torch.cuda.synchronize()
    want = torch.nan_to_num(torch.tensor(OP.decode(*OP.encode(x.double().numpy(), "fp8"), "fp8")), nan=5.5)
    for o in out:
        assert torch.equal(torch.nan_to_num(o.double().cpu(), nan=5.5), want)
    for t, keys in zip(tiles, (True, False)):
        last = t[:, :, -2:].cpu().numpy()
        c, s = OP.from_tiles(last, "fp8", dh, keys)
        assert np.array_equal(c[:, :, -70:], OP.encode(x.double().numpy(), "fp8")[0])


# ---- attention ------------------------------------------------------------------------------------------------------
def sees(p, L, n, sinks, window):
    """[L, n]: which of n rows the queries at p, p + 1, ... see."""
    t, at = torch.arange(n), torch.arange(p, p + L)[:, None]
    return (t <= at) & (torch.tensor(window == 0) | (t < sinks) | (at - t < window))


def make(fmt, dtype, B, L, nh, nkv, dh, P, sinks=0, window=0, starts=None, seed=0, gain=1.0, rows=None):
    rng = np.random.default_rng(seed)
    rows = (P + L + 63) // 64 * 64 if rows is None else rows
    c = dict(q=torch.tensor(rng.normal(size=(B, nh, L, dh)) * gain).to(DT[dtype]), P=P, sinks=sinks, window=window, fmt=fmt, bf16=dtype == "bf16",
             ragged=starts is not None, starts=[min(p, rows - L) for p in (starts or [P] * B)])
    for name, keys in (("k", True), ("v", False)):
        code, scale = OP.encode(rng.normal(size=(B, nkv, rows, dh)) * np.exp(0.5 * rng.normal(size=(1, nkv, 1, dh))), fmt)
        for b, p in enumerate(c["starts"]):      # rows that no query of the call sees hold NaN
            own = np.zeros(rows, bool)
            if p >= 0:
                own[:p + L] = sees(p, L, p + L, sinks, window).any(0).numpy()
            code[b, :, ~own] = 255 if fmt == "fp8" else 15
            scale[b, :, ~own] = 255
        c["t" + name] = torch.tensor(OP.to_tiles(code, scale, fmt, keys))
        c[name] = torch.tensor(OP.decode(code, scale, fmt))
    return c


def plan_of(c, out, q=None, tiles=None, scale=0.0):
    q = c["q"].to(DEV) if q is None else q
    tk, tv = (c["tk"].to(DEV), c["tv"].to(DEV)) if tiles is None else tiles
    P_seq = torch.tensor(c["starts"], dtype=torch.int32, device=DEV) if c["ragged"] else None
    return mulo.make_packed_attention(packed_of(tk, tv, c["fmt"], q.shape[-1]), q, out, c["P"], P_seq=P_seq, sinks=c["sinks"], window=c["window"], scale=scale)


def workspace(plan, fill=0xFF, share=1.0):
    n = int(mulo.mulo_packed_attention_workspace_bytes(plan) * share) // 16 * 16
    return torch.full((n,), fill, dtype=torch.uint8, device=DEV) if n else None      # 0xFF..: NaN


def plain(c, scale=None):
    """The definition with the queries of a sequence side by side, float64, on the device."""
    B, nh, L, dh = c["q"].shape
    group, scale = nh // c["k"].shape[1], dh ** -0.5 if scale is None else scale
    out, mass = torch.zeros(B, nh, L, dh, dtype=torch.float64), torch.zeros(B, nh, L, dh, dtype=torch.float64)
    reach, grouped, keys = torch.zeros(B, nh, L, dtype=torch.float64), torch.zeros(B, nh, L, dtype=torch.float64), torch.zeros(B, L)
    for b, p in enumerate(c["starts"]):
        if p < 0:
            continue
        see = sees(p, L, p + L, c["sinks"], c["window"])
        keys[b] = see.sum(1)
        see = see.to(DEV)
        K, V = (torch.nan_to_num(c[n][b, :, :p + L].to(DEV)) for n in ("k", "v"))      # no query sees the rows of NaN
        for h in range(nh):
            q, Kh, Vh = c["q"][b, h].to(DEV).double(), K[h // group], V[h // group]
            z = (q @ Kh.t().contiguous() * scale).masked_fill(~see, float("-inf"))
            w = torch.exp(z - z.max(-1, keepdim=True).values)
            w = w / w.sum(-1, keepdim=True)
            out[b, h], mass[b, h] = (w @ Vh).cpu(), (w @ Vh.abs()).cpu()
            Ka = Kh.abs().t().contiguous() * scale
            most = q.abs().unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32, -1)
            reach[b, h] = (q.abs() @ Ka).masked_fill(~see, 0.0).max(-1).values.cpu()
            grouped[b, h] = (most @ Ka).masked_fill(~see, 0.0).max(-1).values.cpu()
    return out, mass, reach, keys, grouped


def check(c, out, label, reference):
    want, mass, reach, keys, grouped = reference
    tol = OP.tolerance(mass, reach, keys, want, c["q"].shape[-1], c["bf16"], grouped, torch.nan_to_num(c["v"]).abs().max())
    err = (out.double().cpu() - want).abs()
    assert torch.isfinite(out).all(), "%s: not finite" % label
    worst = (err / (tol + 1e-30)).max().item()
    say("  %s: worst error %.3g of the bound" % (label, worst))
    assert (err <= tol).all(), "%s: %.3g of the bound" % (label, worst)


CASES = [
    # one row; the ends of a tile of rows
    ("fp4", "bf16", 1, 1, 1, 1, 64, 0, {}),
    ("fp4", "bf16", 1, 1, 1, 1, 128, 0, {}),
    ("fp8", "f32", 1, 1, 1, 1, 128, 1, {}),
    ("fp4", "bf16", 2, 1, 2, 2, 128, 62, {}),
    ("fp4", "bf16", 2, 1, 2, 2, 128, 63, {}),
    ("fp8", "bf16", 2, 1, 2, 2, 64, 64, {}),
    ("fp8", "f32", 2, 2, 2, 2, 64, 126, {}),
    ("fp4", "f32", 2, 2, 2, 2, 128, 127, {}),
    # single tokens: shared heads from 2 to 16 and an odd number of them, a long cache
    ("fp4", "bf16", 5, 1, 8, 1, 128, 300, {}),
    ("fp4", "bf16", 3, 1, 16, 1, 64, 700, {}),
    ("fp8", "bf16", 3, 1, 10, 2, 128, 500, {}),
    ("fp8", "bf16", 2, 1, 6, 2, 64, 333, {}),
    ("fp4", "f32", 3, 1, 14, 2, 128, 200, {}),
    ("fp8", "f32", 2, 1, 16, 2, 64, 450, {}),
    ("fp4", "bf16", 1, 1, 2, 2, 128, 5000, {}),
    # a few rows: queries that end inside a block of 16, 32, 64
    ("fp4", "bf16", 2, 5, 4, 4, 128, 100, {}),
    ("fp4", "bf16", 2, 16, 2, 2, 128, 330, {}),
    ("fp8", "bf16", 2, 17, 2, 2, 64, 70, {}),
    ("fp4", "bf16", 2, 9, 8, 2, 64, 128, {}),
    ("fp8", "bf16", 1, 13, 10, 2, 128, 90, {}),
    ("fp4", "bf16", 3, 33, 4, 4, 128, 50, {}),
    ("fp8", "f32", 2, 11, 6, 2, 128, 130, {}),
    ("fp4", "f32", 2, 40, 2, 2, 64, 30, {}),
    # blocks
    ("fp4", "bf16", 2, 130, 4, 1, 64, 11, {}),
    ("fp4", "bf16", 2, 300, 2, 2, 128, 5, {}),
    ("fp8", "bf16", 1, 257, 2, 2, 64, 0, {}),
    ("fp8", "bf16", 1, 190, 4, 2, 128, 700, {}),
    ("fp4", "f32", 1, 150, 4, 2, 128, 9, {}),
    ("fp8", "f32", 1, 260, 2, 2, 64, 0, {}),
    # windows: one row, shorter than a tile, longer than everything, sinks that end inside a tile
    ("fp4", "bf16", 2, 1, 2, 2, 128, 200, dict(window=1)),
    ("fp8", "f32", 2, 7, 2, 2, 64, 200, dict(window=1, sinks=1)),
    ("fp4", "bf16", 3, 5, 4, 2, 128, 300, dict(window=17, sinks=4)),
    ("fp8", "bf16", 2, 1, 2, 2, 64, 3000, dict(window=200, sinks=5)),
    ("fp4", "bf16", 2, 40, 2, 2, 64, 100, dict(window=1000, sinks=3)),
    ("fp4", "bf16", 2, 290, 2, 2, 128, 400, dict(window=130, sinks=70)),
    ("fp8", "bf16", 1, 200, 4, 2, 128, 300, dict(window=90, sinks=130)),
    ("fp4", "f32", 1, 100, 2, 2, 64, 300, dict(window=64, sinks=64)),
    ("fp4", "bf16", 2, 3, 2, 2, 128, 70, dict(window=2 ** 31 - 1, sinks=2 ** 31 - 1)),
    ("fp8", "bf16", 2, 1, 2, 2, 64, 700, dict(window=30, sinks=2 ** 31 - 1)),
    ("fp4", "f32", 1, 140, 2, 2, 64, 70, dict(window=2 ** 31 - 1)),
    # sequences of unequal length, absent ones, one that is longer than the cache allows
    ("fp4", "bf16", 5, 1, 2, 2, 128, 200, dict(starts=[200, 0, -1, 77, 10000])),
    ("fp8", "bf16", 4, 6, 4, 2, 64, 200, dict(starts=[-1, -5, 200, 3], window=60, sinks=7)),
    ("fp8", "f32", 4, 1, 2, 2, 64, 200, dict(starts=[-1, 200, 64, 63])),
    ("fp4", "bf16", 3, 140, 2, 2, 128, 100, dict(starts=[-1, 100, 0])),
    ("fp4", "bf16", 3, 140, 2, 2, 64, 300, dict(starts=[300, 250, 0], window=77, sinks=3)),
    ("fp8", "bf16", 2, 1, 2, 2, 128, 50, dict(starts=[-1, -1])),
    # many sequences and heads; keys dealt to several workgroups
    ("fp4", "bf16", 33, 1, 8, 8, 128, 900, {}),
    ("fp8", "bf16", 16, 1, 32, 8, 128, 1500, dict(starts=[1500, 0, 70, -1, 640, 1499, 1000, 3] * 2)),
    ("fp4", "bf16", 2, 1, 4, 2, 64, 9000, {}),
    ("fp8", "bf16", 1, 16, 8, 2, 128, 4000, dict(window=3500, sinks=33)),
    ("fp4", "f32", 2, 3, 4, 2, 128, 2500, {}),
    ("fp4", "bf16", 4, 64, 8, 8, 128, 1200, {}),
    ("fp4", "bf16", 1, 300, 4, 4, 64, 2000, {}),
    ("fp8", "f32", 1, 70, 4, 4, 64, 1500, dict(starts=[1111])),
]
# Sizes at which keys are dealt to several workgroups or to eight wavefronts, and those of more queries
MANY = [
    # blocks whose wavefronts share a tile's values: whole and ragged tiles of 128 queries, queries that span heads, windows and sinks,
    # sequences of unequal length, absent ones
    ("fp4", "bf16", 5, 150, 32, 32, 128, 33, {}),
    ("fp8", "bf16", 5, 150, 32, 32, 128, 90, dict(starts=[90, 0, -1, 64, 17])),
    ("fp4", "bf16", 8, 128, 32, 32, 128, 0, {}),
    ("fp4", "bf16", 8, 70, 64, 32, 128, 100, dict(window=60, sinks=70)),
    ("fp8", "bf16", 6, 260, 32, 32, 128, 60, dict(window=100, sinks=10)),
    ("fp4", "bf16", 8, 140, 32, 32, 128, 200, dict(window=1, starts=[200, 3, -1, 64, 63, 0, 150, 199])),
    ("fp4", "bf16", 8, 33, 128, 32, 128, 150, dict(starts=[150, -1, 0, 1, 63, 64, 65, 5])),
    ("fp8", "bf16", 16, 150, 32, 32, 64, 40, dict(window=150, sinks=9)),
    ("fp4", "bf16", 16, 128, 32, 32, 64, 70, {}),
    ("fp4", "bf16", 16, 200, 32, 32, 64, 5, dict(starts=[5, -1] * 8)),
    # a few queries over many keys
    ("fp4", "bf16", 2, 1, 8, 8, 128, 3000, {}),
    ("fp8", "bf16", 1, 3, 8, 4, 128, 5000, dict(window=4500, sinks=100)),
    ("fp8", "bf16", 3, 1, 8, 8, 64, 2500, dict(starts=[2500, -1, 700])),
    ("fp4", "bf16", 4, 1, 32, 32, 128, 1100, {}),
    ("fp8", "bf16", 8, 1, 32, 32, 64, 1300, {}),
    ("fp4", "f32", 4, 1, 16, 16, 128, 900, {}),
    ("fp8", "f32", 2, 2, 8, 8, 64, 2100, {}),
    ("fp8", "f32", 4, 40, 8, 8, 64, 600, {}),
    ("fp4", "f32", 6, 90, 16, 16, 64, 200, dict(window=150, sinks=3)),
    ("fp8", "bf16", 12, 40, 32, 32, 128, 300, {}),
    ("fp8", "bf16", 4, 90, 16, 16, 64, 700, {}),
]
# every kernel of every format, type and head size: 32 and 16 queries of a wavefront, four and eight wavefronts, shared values, shares of the keys
EACH = [(fmt, dtype, B, L, nh, nkv, dh, P, dict(kw, starts=[P] + [17] * (B - 1)) if kw else {}) for fmt in ("fp4", "fp8") for dtype in ("bf16", "f32")
        for dh in (64, 128) for B, L, nh, nkv, P in ((2, 200, 32, 8, 30), (4, 200, 32, 8, 30), (1, 200, 4, 1, 30), (1, 17, 4, 1, 1500), (1, 200, 16, 4, 2500))
        for kw in ({}, dict(window=70, sinks=5))]
name_of = lambda c: "%s-%s-%dx%d-h%d.%d-%d-P%d%s" % (c[:8] + ("".join("-%s%s" % (k, v) for k, v in c[8].items() if k != "starts"),))


@pytest.mark.parametrize("case", [CASES[i] for i in (2, 5, 11, 19, 33, 41)], ids=name_of)
def test_plain_form_is_the_oracle(case):
    fmt, dtype, B, L, nh, nkv, dh, P, kw = case
    c = make(fmt, dtype, B, L, nh, nkv, dh, P, **kw)
    got, want = plain(c), OP.packed_attention(c["q"], c["k"], c["v"], c["starts"], c["sinks"], c["window"])
    # Two forms of float64: what the bound of the oracle's module says of float32 with 2^-53 for 2^-24 (and 2^-50 for an exponential's
    # 2^-22), twice, since either may be off.
    out, mass, reach, keys, grouped = got
    rel = 2 * ((dh + 8) * 2.0 ** -53 * reach + 2.0 ** -50) + 2 * (keys[:, None, :] + 8) * 2.0 ** -53
    small = (dh + 8) * 2.0 ** -53
    for a, b, tol in zip((out, mass, reach, grouped), want[:3] + want[4:], (mass * rel[..., None], mass * rel[..., None], small * reach, small * grouped)):
        assert ((a - b).abs() <= 2 * tol).all()
    assert torch.equal(keys, want[3])


@pytest.mark.parametrize("case", CASES + MANY + EACH, ids=name_of)
def test_attention(case):
    fmt, dtype, B, L, nh, nkv, dh, P, kw = case
    c = make(fmt, dtype, B, L, nh, nkv, dh, P, **kw)
    reference = plain(c)
    for share in (1.0, 0.5, 0.0):            # with the scratch it asks for (holding NaN), with less, and with none
        out = torch.full_like(c["q"], NAN, device=DEV)
        plan = plan_of(c, out)
        mulo.mulo_packed_attention(plan, workspace(plan, share=share))
        torch.cuda.synchronize()
        check(c, out, "scratch %g" % share, reference)


@pytest.mark.parametrize("case", [c for c in CASES + MANY if any(p < 0 for p in c[8].get("starts", ()))], ids=name_of)
def test_absent_sequences_are_zeros_whatever_their_queries_hold(case):
    fmt, dtype, B, L, nh, nkv, dh, P, kw = case
    c = make(fmt, dtype, B, L, nh, nkv, dh, P, **kw)
    absent = torch.tensor([p < 0 for p in c["starts"]])
    want = torch.full_like(c["q"], NAN, device=DEV)
    plan = plan_of(c, want)
    mulo.mulo_packed_attention(plan, workspace(plan))
    for bad in (float("inf"), float("-inf"), NAN, torch.finfo(DT[dtype]).max):
        q = c["q"].clone()
        q[absent] = bad
        out = torch.full_like(want, NAN)
        plan = plan_of(c, out, q=q.to(DEV))
        mulo.mulo_packed_attention(plan, workspace(plan))
        torch.cuda.synchronize()
        assert (out[absent.to(DEV)] == 0).all() and torch.equal(out, want), bad


@pytest.mark.parametrize("fmt, dtype, L, dh", [("fp4", "bf16", 4, 128), ("fp8", "bf16", 1, 64), ("fp4", "f32", 4, 64), ("fp8", "f32", 1, 128), ("fp4", "bf16", 150, 128)])
def test_sharp_and_scaled_scores(fmt, dtype, L, dh):
    """Scores of a hundred and more: nearly all of the mass on one row; a scale of the caller's; a query with one loud channel, quiet
    ones and zeros."""
    c = make(fmt, dtype, 3, L, 4, 2, dh, 150, gain=12.0)
    c["q"][0, 0, :, 1:] *= 2.0 ** -9
    c["q"][1, 1, :, ::3] = 0
    c["q"][2, 2] = 0
    c["q"][2, 3] *= 2.0 ** -100
    for scale in (None, 0.25):
        out = torch.full_like(c["q"], NAN, device=DEV)
        plan = plan_of(c, out, scale=scale or 0.0)
        mulo.mulo_packed_attention(plan, workspace(plan))
        torch.cuda.synchronize()
        check(c, out, "scale %s" % scale, plain(c, scale))


@pytest.mark.parametrize("fmt, dtype", [("fp4", "bf16"), ("fp8", "f32")])
@pytest.mark.parametrize("size", [1e-30, 1e30])
def test_very_large_and_very_small_numbers(fmt, dtype, size):
    """Keys of either size against queries of the other, values of either."""
    c = make(fmt, dtype, 2, 3, 4, 2, 64, 100)
    e = round(np.log2(size))
    for name, keys in (("k", True), ("v", False)):
        code, scale = OP.from_tiles(c["t" + name].numpy(), fmt, 64, keys)
        scale = np.where(scale == 255, 255, scale.astype(int) + e).astype(np.uint8)
        c["t" + name] = torch.tensor(OP.to_tiles(code, scale, fmt, keys))
        c[name] = torch.tensor(OP.decode(code, scale, fmt))
    c["q"] = (c["q"].double() * 2.0 ** -e).to(c["q"].dtype)
    out = torch.full_like(c["q"], NAN, device=DEV)
    plan = plan_of(c, out)
    mulo.mulo_packed_attention(plan, workspace(plan))
    torch.cuda.synchronize()
    check(c, out, "numbers of %g" % size, plain(c))


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype, B, L, nh, nkv, dh, P", [
    ("bf16", 3, 1, 4, 2, 128, 100), ("bf16", 2, 20, 4, 4, 64, 90), ("bf16", 2, 1, 4, 2, 64, 3000), ("bf16", 8, 128, 32, 32, 128, 0), ("bf16", 16, 128, 32, 32, 64, 70),
    ("f32", 3, 1, 4, 2, 128, 100), ("f32", 2, 20, 4, 4, 64, 90), ("f32", 2, 1, 4, 2, 64, 3000)])
def test_queries_at_the_end_of_their_type(fmt, dtype, B, L, nh, nkv, dh, P):
    """The largest numbers a query can hold against the smallest keys of a cache, so that the scores are ordinary numbers (the queries'
    2^128, the keys' 2^-117 and a scale of 2^-14).  Whole queries from 0.9 of the largest number up, and queries with the largest one
    beside ordinary numbers."""
    c = make(fmt, dtype, B, L, nh, nkv, dh, P)
    code, scale = OP.from_tiles(c["tk"].numpy(), fmt, dh, True)
    scale = np.where(scale == 255, 255, 10).astype(np.uint8)
    if fmt == "fp8":      # up to 7.5
        code = np.where((code & 127) < 0x50, code, code & 0x80 | code & 7 | 0x48).astype(np.uint8)
        code[scale.repeat(32, -1) == 255] = 255
    c["tk"], c["k"] = torch.tensor(OP.to_tiles(code, scale, fmt, True)), torch.tensor(OP.decode(code, scale, fmt))
    top = torch.finfo(DT[dtype]).max
    g = torch.Generator().manual_seed(7)
    q = ((0.9 + 0.1 * torch.rand(c["q"].shape, generator=g, dtype=torch.float64)) * top * (1 - 2 * torch.randint(0, 2, c["q"].shape, generator=g))).clamp(-top, top)
    q[0, ::2] = torch.randn(q[0, ::2].shape, generator=g, dtype=torch.float64)
    q[0, ::2, :, 0], q[0, ::2, :, dh - 1] = top, -top
    c["q"] = q.to(DT[dtype])
    assert torch.isfinite(c["q"]).all() and (c["q"].abs() == top).any()
    out = torch.full_like(c["q"], NAN, device=DEV)
    plan = plan_of(c, out, scale=2.0 ** -14)
    mulo.mulo_packed_attention(plan, workspace(plan))
    torch.cuda.synchronize()
    check(c, out, "queries up to %g" % top, plain(c, 2.0 ** -14))


@pytest.mark.parametrize("L", [1, 20, 150])
def test_strides(L):
    """Token-major queries and output inside a wider row, a cache whose heads lie in front of its sequences and inside a larger one; what
    lies around the output stays as it was."""
    B, nh, nkv, dh = 3, 4, 2, 64
    c = make("fp4", "bf16", B, L, nh, nkv, dh, 40)
    wide = torch.full((B, L, nh + 2, dh), 7.0, dtype=torch.bfloat16, device=DEV)
    out = wide[:, :, 1:nh + 1].permute(0, 2, 1, 3)
    q = torch.zeros(B, L, nh, 2 * dh, dtype=torch.bfloat16, device=DEV)
    q[..., :dh] = c["q"].permute(0, 2, 1, 3).to(DEV)
    tiles = []
    for name in ("tk", "tv"):
        n, size = c[name].shape[2:]
        w = torch.full((nkv + 1, B, n + 3, size), 255, dtype=torch.uint8, device=DEV)
        w[1:, :, 2:2 + n] = c[name].transpose(0, 1).to(DEV)
        tiles.append(w[1:, :, 2:2 + n].transpose(0, 1))
    plan = plan_of(c, out, q=q[..., :dh].permute(0, 2, 1, 3), tiles=tiles)
    mulo.mulo_packed_attention(plan, workspace(plan))
    torch.cuda.synchronize()
    check(c, out, "strided", plain(c))
    assert (wide[:, :, 0] == 7).all() and (wide[:, :, nh + 1] == 7).all()


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_sequences_that_share_a_cache(fmt):
    """A batch stride of 0: drafts of one picture over the same rows."""
    c = make(fmt, "bf16", 1, 3, 4, 2, 128, 200)
    tiles = [c[n].to(DEV).expand(5, -1, -1, -1) for n in ("tk", "tv")]
    c["q"] = torch.randn(5, 4, 3, 128, generator=torch.Generator().manual_seed(8)).bfloat16()
    c["k"], c["v"], c["starts"] = c["k"].expand(5, -1, -1, -1), c["v"].expand(5, -1, -1, -1), [200] * 5
    out = torch.full_like(c["q"], NAN, device=DEV)
    plan = plan_of(c, out, tiles=tiles)
    mulo.mulo_packed_attention(plan, workspace(plan))
    torch.cuda.synchronize()
    check(c, out, "shared", plain(c))


@pytest.mark.parametrize("fmt, dtype", [("fp8", "bf16"), ("fp4", "f32")])
def test_offsets_beyond_32_bits(fmt, dtype):
    """The last rows of a cache whose heads are longer than 2^31 and 2^30 bytes: the same as those rows on their own."""
    rows, n, dh = 1 << 24, 320, 128
    g = torch.Generator().manual_seed(3)
    tiles = [torch.empty(1, 3, rows // 64, OP.tile_bytes(fmt, dh), dtype=torch.uint8, device=DEV) for _ in range(2)]
    short = [torch.empty(1, 3, n // 64 + 1, OP.tile_bytes(fmt, dh), dtype=torch.uint8, device=DEV) for _ in range(2)]
    for (first, many) in ((0, 64), (rows - n, n)):
        x = [torch.randn(1, 3, many, dh, generator=g).to(DT[dtype]).to(DEV) for _ in range(2)]
        mulo.mulo_pack_rows(packed_of(*tiles, fmt, dh), mulo.make_kv_rows(*x, first))
        mulo.mulo_pack_rows(packed_of(*short, fmt, dh), mulo.make_kv_rows(*x, 64 if first else 0))
    for L in (1, 140):
        q = torch.randn(1, 6, L, dh, generator=g).to(DT[dtype]).to(DEV)
        outs = []
        for t, P in ((tiles, rows - L), (short, n + 64 - L)):
            out = torch.empty_like(q)
            plan = mulo.make_packed_attention(packed_of(*t, fmt, dh), q, out, P, sinks=8, window=150)
            mulo.mulo_packed_attention(plan, workspace(plan))
            outs.append(out)
        torch.cuda.synchronize()
        assert torch.isfinite(outs[0]).all() and torch.equal(*outs)


@pytest.mark.parametrize("fmt, dtype, L", [("fp4", "bf16", 1), ("fp8", "bf16", 20), ("fp4", "f32", 3)])
def test_bits_do_not_depend_on_the_workspace_or_the_run(fmt, dtype, L):
    c = make(fmt, dtype, 4, L, 8, 4, 128, 1500)
    outs = []
    for fill in (0, 0xFF, 0x7F):
        out = torch.full_like(c["q"], NAN, device=DEV)
        plan = plan_of(c, out)
        mulo.mulo_packed_attention(plan, workspace(plan, fill))
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("fmt, nh", [("fp4", 4), ("fp8", 16)])
def test_a_decoding_loop_recorded_once(fmt, nh):
    """One graph packs a token's rows and attends to the cache: the lengths live on the device.  Every replay against eager calls on a
    cache of their own and against the definition."""
    B, nkv, dh, P = 5, 4, 128, 300
    g = torch.Generator().manual_seed(1)
    normal = lambda *s: torch.randn(*s, generator=g).bfloat16().to(DEV)
    caches = [mulo.alloc_packed_kv(B, nkv, P + 1, dh, FMT[fmt], DEV) for _ in range(2)]
    fill = [normal(B, nkv, P + 1, dh) for _ in range(2)]
    for cache in caches:
        mulo.mulo_pack_rows(cache, mulo.make_kv_rows(*fill, 0))
    k, v, q = normal(B, nkv, 1, dh), normal(B, nkv, 1, dh), normal(B, nh, 1, dh)
    P_seq = torch.zeros(B, dtype=torch.int32, device=DEV)
    rows = mulo.make_kv_rows(k, v, P, P_seq)
    outs = [torch.empty_like(q) for _ in range(2)]
    plans = [mulo.make_packed_attention(cache, q, out, P, P_seq=P_seq) for cache, out in zip(caches, outs)]
    spaces = [workspace(p) for p in plans]

    def step(i):
        mulo.mulo_pack_rows(caches[i], rows)
        mulo.mulo_packed_attention(plans[i], spaces[i])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(1)
        side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(0)
    with torch.cuda.stream(side):
        for cache in caches:
            mulo.mulo_pack_rows(cache, mulo.make_kv_rows(*fill, 0))
        for rep, lens in enumerate(([0, 1, 2, 63, 64], [300, 299, -1, 5, 100], [7] * 5, [8] * 5, [300] * 5)):
            P_seq.copy_(torch.tensor(lens, dtype=torch.int32))
            for t in (k, v, q):
                t.copy_(normal(*t.shape))
            graph.replay()
            step(1)
            side.synchronize()
            assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v) and torch.equal(*outs), rep
            tiles = [t.cpu().numpy() for t in (caches[0].k, caches[0].v)]
            c = dict(q=q.cpu(), starts=lens, sinks=0, window=0, bf16=True)
            c["k"], c["v"] = (torch.tensor(OP.decode(*OP.from_tiles(t, fmt, dh, keys), fmt)) for t, keys in zip(tiles, (True, False)))
            check(c, outs[0], "replay %d" % rep, plain(c))
    del graph


def test_on_a_stream_of_the_callers():
    """Work on another stream than the current one, given as a raw stream."""
    c = make("fp4", "bf16", 2, 4, 4, 2, 128, 900)
    out = torch.full_like(c["q"], NAN, device=DEV)
    plan = plan_of(c, out)
    ws = workspace(plan)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mulo.mulo_packed_attention(plan, ws, stream=side.cuda_stream)
    side.synchronize()
    check(c, out, "side stream", plain(c))


# ---- together, as a context's cache goes in and out --------------------------------------------------------------------
def small_context(B, max_seq, block):
    from workloads import configs as WC
    from workloads import generators as WG
    m = dict(WC.model("small"), n_layers=2)
    w = WG.make_weights(m, seed=0)
    cos, sin = WG.rope_table(max_seq, m["head_dim"])
    cfg = mulo.make_cfg(m, B, max_seq, block)
    ctx = mulo.mulo_create(cfg, {k: t.to(DEV) for k, t in w.items()}, torch.tensor(cos, device=DEV), torch.tensor(sin, device=DEV))
    return m, ctx


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_a_contexts_cache_packed_attended_and_restored(fmt):
    """A context's prompt rows go into a packed cache, layer by layer; attention over them is attention over what comes back; a context
    that gets them back goes on with the numbers that the packed cache stands for."""
    B, P, max_seq = 2, 150, 192
    m, ctx = small_context(B, max_seq, max(P, 4) + 2)
    nl, nh, dh, V = m["n_layers"], m["n_heads"], m["head_dim"], m["vocab"]
    kv = mulo.alloc_kv(ctx, DEV)
    g = torch.Generator().manual_seed(4)
    tokens = torch.randint(0, V, (B, P), generator=g, dtype=torch.int32).to(DEV)
    mulo.mulo_verify_forward(ctx, kv, B, P, 0, tokens, None, torch.empty(B, P, V, device=DEV))
    back = mulo.alloc_kv(ctx, DEV)
    q = torch.randn(B, nh, 3, dh, generator=g).bfloat16().to(DEV)
    for layer in range(nl):
        packed = mulo.alloc_packed_kv(B, nh, P, dh, FMT[fmt], DEV)
        of = lambda c: (c[0][layer][:, :, :P], c[1][layer][:, :, :, :P].transpose(2, 3))
        mulo.mulo_pack_rows(packed, mulo.make_kv_rows(*of(kv), 0))
        mulo.mulo_unpack_rows(packed, mulo.make_kv_rows(*of(back), 0))
        torch.cuda.synchronize()
        for x, y in zip(of(kv), of(back)):
            want = OP.decode(*OP.encode(x.double().cpu().numpy(), fmt), fmt)
            assert np.array_equal(y.double().cpu().numpy(), want)
        # the same attention over the packed rows and over what the other cache holds
        outs = [torch.empty_like(q) for _ in range(2)]
        plan = mulo.make_packed_attention(packed, q, outs[0], P - 3)
        mulo.mulo_packed_attention(plan, workspace(plan))
        other = mulo.make_attention(q, outs[1], back[0][layer], back[1][layer], P - 3)
        mulo.mulo_attention(other)
        torch.cuda.synchronize()
        c = dict(q=q.cpu(), starts=[P - 3] * B, sinks=0, window=0, bf16=True, k=of(back)[0].double().cpu(), v=of(back)[1].double().cpu())
        reference = plain(c)
        check(c, outs[0], "packed", reference)
        check(c, outs[1], "unpacked", reference)
    # the context goes on from the restored rows as from a cache that was filled with the same numbers
    nxt = torch.randint(0, V, (B, 1), generator=g, dtype=torch.int32).to(DEV)
    copy = tuple(t.clone() for t in back)
    logits = [torch.empty(B, 1, V, device=DEV) for _ in range(3)]
    mulo.mulo_verify_forward(ctx, back, B, 1, P, nxt, None, logits[0])
    mulo.mulo_verify_forward(ctx, copy, B, 1, P, nxt, None, logits[1])
    mulo.mulo_verify_forward(ctx, kv, B, 1, P, nxt, None, logits[2])
    torch.cuda.synchronize()
    assert torch.isfinite(logits[0]).all() and torch.equal(logits[0], logits[1])
    say("  logits of the next token, %s cache against bf16: relative 2-norm of the difference %.3g" % (fmt, ((logits[0] - logits[2]).norm() / logits[2].norm()).item()))


# ---- calls that a careless program makes -------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt, dtype, B, L, nh, nkv, dh, P", [
    ("fp4", "bf16", 2, 1, 8, 2, 128, 300), ("fp8", "bf16", 2, 1, 4, 1, 64, 2500), ("fp4", "bf16", 8, 128, 32, 32, 128, 0), ("fp8", "bf16", 2, 70, 4, 4, 64, 90),
    ("fp4", "f32", 2, 5, 8, 4, 128, 200), ("fp8", "f32", 2, 40, 4, 4, 64, 100)])
def test_a_query_that_is_not_finite_spoils_its_own_output(fmt, dtype, B, L, nh, nkv, dh, P):
    c = make(fmt, dtype, B, L, nh, nkv, dh, P)
    want = torch.full_like(c["q"], NAN, device=DEV)
    plan = plan_of(c, want)
    mulo.mulo_packed_attention(plan, workspace(plan))
    b, h, j = B - 1, nh // 2, L // 2
    keep = torch.ones(B, nh, L, dtype=torch.bool, device=DEV)
    keep[b, h, j] = False
    for bad in (NAN, float("inf"), float("-inf")):
        for channel in (0, dh - 1):
            q = c["q"].clone()
            q[b, h, j, channel] = bad
            out = torch.full_like(want, 7.0)
            plan = plan_of(c, out, q=q.to(DEV))
            mulo.mulo_packed_attention(plan, workspace(plan))
            torch.cuda.synchronize()
            assert torch.equal(out[keep], want[keep]), (bad, channel)


@pytest.mark.parametrize("fmt, dtype, B, L, nh, nkv, dh, P, shares", [
    ("fp4", "bf16", 2, 1, 8, 2, 128, 300, False), ("fp4", "bf16", 8, 128, 32, 32, 128, 0, False), ("fp8", "bf16", 2, 70, 4, 4, 64, 90, False),
    ("fp4", "f32", 2, 5, 8, 4, 128, 200, False), ("fp8", "f32", 2, 40, 4, 4, 64, 100, False),
    ("fp8", "bf16", 2, 1, 4, 1, 64, 2500, True), ("fp4", "bf16", 2, 3, 8, 2, 128, 4000, True), ("fp4", "f32", 2, 3, 4, 2, 128, 2500, True), ("fp8", "f32", 2, 2, 8, 8, 64, 3000, True)])
def test_a_query_that_is_not_finite_is_answered_with_nan(fmt, dtype, B, L, nh, nkv, dh, P, shares):
    """All of its channels, also where its keys are dealt to several workgroups."""
    c = make(fmt, dtype, B, L, nh, nkv, dh, P)
    b, h, j = B - 1, nh // 2, L // 2
    for bad in (NAN, float("inf"), float("-inf")):
        q = c["q"].clone()
        q[b, h, j, 1] = bad
        out = torch.full_like(q, 7.0, device=DEV)
        plan = plan_of(c, out, q=q.to(DEV))
        assert (mulo.mulo_packed_attention_workspace_bytes(plan) > 0) == shares
        for ws in (workspace(plan, 0), None):
            mulo.mulo_packed_attention(plan, ws)
            torch.cuda.synchronize()
            nans = torch.isnan(out).sum(-1).tolist()
            assert nans[b][h][j] == dh and np.sum(nans) == dh, bad


def test_keys_and_values_out_of_one_tensor():
    """Heads of one cache, and of one tensor of rows: next to each other and in turn they are written, on top of each other they are not."""
    B, nkv, L, dh, rows = 2, 2, 5, 64, 64
    g = torch.Generator().manual_seed(2)
    x = [torch.randn(B, nkv, L, dh, generator=g).bfloat16() for _ in range(2)]
    size = OP.tile_bytes("fp4", dh)
    both = lambda t, how: (t[:, :nkv], t[:, nkv:2 * nkv]) if how == "next" else (t[:, 0:2 * nkv:2], t[:, 1:2 * nkv:2]) if how == "in turn" else (t[:, :nkv], t[:, 1:nkv + 1])
    row_in = mulo.make_kv_rows(*(t.to(DEV) for t in x), 3)
    want = [torch.tensor(OP.decode(*OP.encode(t.double().numpy(), "fp4"), "fp4")) for t in x]
    for cache_how in ("next", "in turn"):
        tiles = torch.zeros(B, 2 * nkv, rows // 64, size, dtype=torch.uint8, device=DEV)
        packed = packed_of(*both(tiles, cache_how), "fp4", dh)
        mulo.mulo_pack_rows(packed, row_in)
        for how in ("next", "in turn"):
            big = torch.full((B, 2 * nkv, L, dh), NAN, dtype=torch.bfloat16, device=DEV)
            out = both(big, how)
            mulo.mulo_unpack_rows(packed, mulo.make_kv_rows(*out, 3))
            torch.cuda.synchronize()
            assert all(torch.equal(o.double().cpu(), w) for o, w in zip(out, want)), (cache_how, how)
        before = big.clone()
        with pytest.raises(mulo.MuloError):
            mulo.mulo_unpack_rows(packed, mulo.make_kv_rows(*both(big, "shifted"), 3))
        assert torch.equal(big, before)
    before = tiles.clone()
    with pytest.raises(mulo.MuloError):
        mulo.mulo_pack_rows(packed_of(*both(tiles, "shifted"), "fp4", dh), row_in)
    assert torch.equal(tiles, before)


@pytest.mark.parametrize("fmt, dtype, L", [("fp4", "bf16", 1), ("fp8", "f32", 7), ("fp4", "bf16", 140)])
def test_the_lowest_and_the_highest_starts(fmt, dtype, L):
    """Starts at either end of the type: absent, and the last rows that there are."""
    B, nkv, dh, rows = 4, 2, 64, 192
    low, high = -2 ** 31, 2 ** 31 - 1
    starts = torch.tensor([low, high, 0, low], dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(6)
    tiles = [torch.full((B, nkv, rows // 64, OP.tile_bytes(fmt, dh)), 0x2A, dtype=torch.uint8, device=DEV) for _ in range(2)]
    before = tiles[0].clone()
    x = [torch.randn(B, nkv, L, dh, generator=g).to(DT[dtype]).to(DEV) for _ in range(2)]
    packed = packed_of(*tiles, fmt, dh)
    mulo.mulo_pack_rows(packed, mulo.make_kv_rows(*x, rows - L, starts))
    back = [torch.full_like(y, 5.0) for y in x]
    mulo.mulo_unpack_rows(packed, mulo.make_kv_rows(*back, rows - L, starts))
    torch.cuda.synchronize()
    for t in tiles:
        assert torch.equal(t[[0, 3]], before[[0, 3]])
    for y, z in zip(x, back):
        want = torch.tensor(OP.decode(*OP.encode(y.double().cpu().numpy(), fmt), fmt)).to(DT[dtype])
        assert torch.equal(z[[1, 2]].cpu(), want[[1, 2]]) and (z[[0, 3]] == 5).all()
    q = torch.randn(B, 4, L, dh, generator=g).to(DT[dtype]).to(DEV)
    clamped = torch.tensor([-1, rows - L, 0, -1], dtype=torch.int32, device=DEV)
    for window in (0, 30):
        outs = []
        for s in (starts, clamped):
            out = torch.full_like(q, NAN)
            plan = mulo.make_packed_attention(packed, q, out, rows - L, P_seq=s, window=window, sinks=3)
            mulo.mulo_packed_attention(plan, workspace(plan))
            outs.append(out)
        torch.cuda.synchronize()
        assert torch.isfinite(outs[0]).all() and torch.equal(*outs) and (outs[0][[0, 3]] == 0).all()


def test_two_graphs_on_two_streams():
    """Two recorded calls, each with scratch of its own, replayed beside each other and beside eager calls."""
    cs = [make(fmt, "bf16", 2, 1, 8, 8, 128, P) for fmt, P in (("fp4", 3000), ("fp8", 2500))]
    wants, outs, plans, spaces, graphs, sides = [], [], [], [], [], []
    for c in cs:
        want = torch.full_like(c["q"], NAN, device=DEV)
        plan = plan_of(c, want)
        mulo.mulo_packed_attention(plan, workspace(plan))
        wants.append(want)
        out = torch.full_like(want, NAN)
        plan = plan_of(c, out)
        plans.append(plan)
        spaces.append(workspace(plan))
        outs.append(out)
        sides.append(torch.cuda.Stream())
    torch.cuda.synchronize()
    assert all(mulo.mulo_packed_attention_workspace_bytes(p) for p in plans)
    for plan, ws, side in zip(plans, spaces, sides):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            mulo.mulo_packed_attention(plan, ws)
        graphs.append(graph)
    for rep in range(4):
        for out in outs:
            out.fill_(NAN)
        torch.cuda.synchronize()
        for graph, side in zip(graphs, sides):
            with torch.cuda.stream(side):
                for _ in range(3):
                    graph.replay()
        eager = torch.full_like(wants[0], NAN)
        plan = plan_of(cs[0], eager)
        mulo.mulo_packed_attention(plan, workspace(plan))
        torch.cuda.synchronize()
        assert torch.equal(outs[0], wants[0]) and torch.equal(outs[1], wants[1]) and torch.equal(eager, wants[0]), rep
    del graphs
