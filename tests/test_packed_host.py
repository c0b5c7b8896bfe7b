"""CPU-side checks of mulo_pack_rows, mulo_unpack_rows and mulo_packed_attention: what they refuse, before anything touches a GPU,
and their oracle's own pins."""
import ctypes as C
import math
import os
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2601_05149_amd as mulo
from oracle import packed as OP
from paper_2601_05149_amd import binding as BD

NULL, SHAPE, RANGE, UNSUPPORTED = 1, 2, 3, 6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(BD.LIB_PATH):
        from paper_2601_05149_amd import build
        build.build_lib()
    return mulo.load_library()


# 4 sequences of 2 heads of 64, 128 rows in 4 bits: tiles of 2176 bytes
HEAD = 2 * 2176
KV = dict(format=0, B=4, n_kv_heads=2, head_dim=64, rows=128, k=1 << 20, v=1 << 21, batch=2 * HEAD, head=HEAD)
ROWS = dict(dtype=1, L=3, k=256, v=512, k_batch=384, k_head=192, k_row=64, v_batch=384, v_head=192, v_row=64, v_chan=1, P=125)
ACROSS = dict(v_row=1, v_chan=3, v_head=192, v_batch=384)


def split(changes):
    kv, rows = dict(KV), dict(ROWS)
    for name, value in changes.items():
        (kv if name in ("format", "B", "n_kv_heads", "head_dim", "rows", "pk", "pv", "batch", "head") else rows)[name[1:] if name in ("pk", "pv") else name] = value
    return BD.PackedKV(**kv), BD.KVRows(**rows)


@pytest.mark.parametrize("fmt, dh, size", [(0, 128, 64 * 68), (0, 64, 64 * 34), (1, 128, 64 * 132), (1, 64, 64 * 66), (2, 64, 0), (-1, 64, 0), (0, 96, 0)])
def test_tile_bytes(lib, fmt, dh, size):
    assert mulo.mulo_packed_tile_bytes(fmt, dh) == size
    if size:
        assert OP.tile_bytes(["fp4", "fp8"][fmt], dh) == size


# status of packing, and of unpacking where that is another
@pytest.mark.parametrize("status, other, changes", [
    (NULL, NULL, dict(k=None, v=None)), (NULL, NULL, dict(pk=None)), (NULL, NULL, dict(pv=None)),
    (RANGE, RANGE, dict(dtype=2)), (RANGE, RANGE, dict(L=0)), (RANGE, RANGE, dict(P=-1)), (RANGE, RANGE, dict(format=2)), (RANGE, RANGE, dict(B=0)),
    (RANGE, RANGE, dict(n_kv_heads=0)), (RANGE, RANGE, dict(head_dim=0)), (RANGE, RANGE, dict(rows=0)), (RANGE, RANGE, dict(batch=-16)), (RANGE, RANGE, dict(head=1 << 41)),
    (RANGE, RANGE, dict(k_row=-8)), (RANGE, RANGE, dict(v_batch=1 << 41)),
    (SHAPE, SHAPE, dict(P=126)), (SHAPE, SHAPE, dict(P=2 ** 31 - 1)), (SHAPE, SHAPE, dict(pv=1 << 20)),
    (UNSUPPORTED, UNSUPPORTED, dict(head_dim=96)), (UNSUPPORTED, UNSUPPORTED, dict(rows=96, P=0)), (UNSUPPORTED, UNSUPPORTED, dict(rows=(1 << 24) + 64)),
    (UNSUPPORTED, UNSUPPORTED, dict(batch=2 * HEAD + 8)), (UNSUPPORTED, UNSUPPORTED, dict(head=HEAD + 8)), (UNSUPPORTED, UNSUPPORTED, dict(pk=(1 << 20) + 8)),
    (UNSUPPORTED, UNSUPPORTED, dict(pv=(1 << 21) + 4)), (UNSUPPORTED, UNSUPPORTED, dict(k=264)), (UNSUPPORTED, UNSUPPORTED, dict(k_row=68)),
    (UNSUPPORTED, UNSUPPORTED, dict(v=520)), (UNSUPPORTED, UNSUPPORTED, dict(v_head=196)), (UNSUPPORTED, UNSUPPORTED, dict(v_chan=2)),
    (UNSUPPORTED, UNSUPPORTED, dict(ACROSS, v=513)), (UNSUPPORTED, UNSUPPORTED, dict(dtype=0, k_row=66)),
    (UNSUPPORTED, UNSUPPORTED, dict(B=1 << 22, P=0, L=1)), (UNSUPPORTED, UNSUPPORTED, dict(B=1 << 20, L=33, P=0, k_head=2112, v_head=2112, k_batch=4224, v_batch=4224)),
    # a cache whose tiles lie on top of each other is not written
    (SHAPE, 0, dict(batch=HEAD)), (SHAPE, 0, dict(head=HEAD - 16)), (SHAPE, 0, dict(batch=0)),
    # nor rows of numbers
    (0, SHAPE, dict(k_batch=0)), (0, SHAPE, dict(k_row=0)), (0, SHAPE, dict(v_head=64)), (0, SHAPE, dict(v=256)), (0, SHAPE, dict(dtype=0, k_head=188)),
    (0, SHAPE, dict(ACROSS, v_head=189)), (0, SHAPE, dict(ACROSS, v_chan=2)),
], ids=str)
def test_rows_arguments(lib, status, other, changes):
    kv, r = split(changes)
    both = status if status == other else 0
    assert lib.mulo_check_packed_rows(C.byref(kv), C.byref(r)) == both
    if status:
        assert lib.mulo_pack_rows(None, C.byref(kv), C.byref(r)) == status
    if other:
        assert lib.mulo_unpack_rows(None, C.byref(kv), C.byref(r)) == other


@pytest.mark.parametrize("changes", [
    {}, dict(k=None, pk=None), dict(v=None, pv=None), dict(dtype=0), ACROSS, dict(ACROSS, v=514), dict(v_chan=999, v_row=0, v_batch=1 << 20, v_head=1 << 18, L=1),
    dict(batch=HEAD, head=4 * HEAD), dict(B=1, batch=0), dict(B=1 << 21, P=0, L=16, batch=2 * HEAD), dict(format=1, head_dim=128, batch=1 << 20, head=1 << 16)], ids=str)
def test_rows_arguments_that_hold(lib, changes):
    kv, r = split(changes)
    assert lib.mulo_check_packed_rows(C.byref(kv), C.byref(r)) == 0


def test_rows_without_arguments(lib):
    kv, r = split({})
    for call in (lib.mulo_check_packed_rows, lambda a, b: lib.mulo_pack_rows(None, a, b), lambda a, b: lib.mulo_unpack_rows(None, a, b)):
        assert call(None, C.byref(r)) == NULL and call(C.byref(kv), None) == NULL


def attention_args(**changes):
    kv = dict(KV)
    a = dict(dtype=1, L=2, n_heads=8, q=256, q_batch=1024, q_head=128, q_row=64, out=512, out_batch=1024, out_head=64, out_row=512, P=126,
             sinks=3, window=9, scale=0.0)
    for name, value in changes.items():
        if name in ("pk", "pv"):
            kv[name[1:]] = value
        else:
            (kv if name in kv else a)[name] = value
    return BD.PackedAttentionArgs(kv=BD.PackedKV(**kv), **a)


@pytest.mark.parametrize("status, changes", [
    (0, {}), (0, dict(window=0)), (0, dict(sinks=2 ** 31 - 1, window=2 ** 31 - 1)), (0, dict(batch=0, head=0)), (0, dict(format=1)), (0, dict(dtype=0)),
    (NULL, dict(q=None)), (NULL, dict(out=None)), (NULL, dict(pk=None)), (NULL, dict(pv=None)),
    (RANGE, dict(dtype=2)), (RANGE, dict(format=3)), (RANGE, dict(B=0)), (RANGE, dict(L=0)), (RANGE, dict(n_heads=0)), (RANGE, dict(n_kv_heads=0)), (RANGE, dict(P=-1)),
    (RANGE, dict(rows=0)), (RANGE, dict(sinks=-1)), (RANGE, dict(window=-1)), (RANGE, dict(scale=-1.0)), (RANGE, dict(scale=math.nan)),
    (RANGE, dict(scale=math.inf)), (RANGE, dict(q_batch=-8)), (RANGE, dict(out_row=1 << 41)), (RANGE, dict(batch=-16)),
    (SHAPE, dict(P=127)), (SHAPE, dict(n_heads=7)), (SHAPE, dict(pv=1 << 20)),
    (SHAPE, dict(out_batch=0)), (SHAPE, dict(out_head=32)), (SHAPE, dict(out_row=64)), (SHAPE, dict(out_batch=512)), (0, dict(L=1, out_row=0)),
    (UNSUPPORTED, dict(head_dim=32)), (UNSUPPORTED, dict(q_row=68)), (UNSUPPORTED, dict(rows=100, P=0)), (UNSUPPORTED, dict(q=264)), (UNSUPPORTED, dict(out=8)),
    (UNSUPPORTED, dict(head=8)), (UNSUPPORTED, dict(pk=4100)), (UNSUPPORTED, dict(dtype=0, q_row=66)), (0, dict(dtype=0, q_row=68)),
    (UNSUPPORTED, dict(B=1 << 20)), (0, dict(B=1 << 19)), (UNSUPPORTED, dict(B=1 << 19, L=16, P=0, out_batch=8192)), (0, dict(B=1 << 18, L=16, P=0, out_batch=8192)),
], ids=str)
def test_attention_arguments(lib, status, changes):
    a = attention_args(**changes)
    assert lib.mulo_check_packed_attention(C.byref(a)) == status
    if status:
        assert lib.mulo_packed_attention(None, C.byref(a), None, 0) == status
        assert lib.mulo_packed_attention_workspace_bytes(C.byref(a)) == 0


def test_attention_without_arguments(lib):
    assert lib.mulo_check_packed_attention(None) == NULL and lib.mulo_packed_attention(None, None, None, 0) == NULL
    assert lib.mulo_packed_attention(None, C.byref(attention_args()), C.c_void_p(8), 64) == UNSUPPORTED       # a workspace off its 16 bytes


# ---- the oracle ------------------------------------------------------------------------------------------------------
def test_grids():
    assert OP.grid("fp4").tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    g = OP.grid("fp8")
    assert len(g) == 127 and g[1] == 2.0 ** -9 and g[-1] == 448 and (np.diff(g) > 0).all()
    import torch as T
    if hasattr(T, "float8_e4m3fn"):      # the library's own type
        assert np.array_equal(g, T.arange(127, dtype=T.uint8).view(T.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_codes_by_exact_arithmetic(fmt):
    """Against fractions: the smallest exponent that reaches, and no number of the grid nearer than the one that was taken."""
    f, G = OP.FORMATS[fmt], [Fraction(float(x)) for x in OP.grid(fmt)]
    rng = np.random.default_rng(0)
    x = rng.normal(size=(12, 32)).astype(np.float32) * (10.0 ** rng.integers(-30, 30, (12, 1))).astype(np.float32)
    x[0] = 0
    x[1, :4], x[1, 4:] = [7, -7, 464, 1], 0.25      # what a group may just reach
    x[2], x[3] = np.float32(2.0 ** -140), np.float32(3.4e38)
    x[4, :16], x[4, 16:] = np.tile([0.25, -0.75, 1.25, -1.75, 2.5, -3.5, 5, -6.5], 2), 7
    code, scale = OP.encode(x, fmt)
    back = OP.decode(code, scale, fmt)
    for row, cs, s, ys in zip(x, code, scale, back):
        m, e = max(abs(Fraction(float(v))) for v in row), int(s[0]) - 127
        fits = lambda n: m <= Fraction(f["reach"]) * Fraction(2) ** n
        assert -117 <= e <= f["cap"] and (fits(e) or e == f["cap"]) and (e == -117 or not fits(e - 1))
        for v, c, y in zip(row, cs, ys):
            a, c = abs(Fraction(float(v))) / Fraction(2) ** e, int(c) % (1 << (f["bits"] - 1))
            off = abs(a - G[c])
            assert all(off < abs(a - g) or (off == abs(a - g) and (c % 2 == 0 or c == i)) for i, g in enumerate(G) if i != c)
            assert Fraction(float(y)) == (G[c] if v >= 0 else -G[c]) * Fraction(2) ** e
            if e < f["cap"]:      # half of the widest step
                assert off <= (1 if fmt == "fp4" else 16)


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_numbers_that_are_none(fmt):
    x = np.ones((2, 64), np.float32)
    x[0, 3], x[1, 40] = np.nan, -np.inf
    code, scale = OP.encode(x, fmt)
    assert (scale == 255).tolist() == [[True, False], [False, True]]
    back = OP.decode(code, scale, fmt)
    assert np.isnan(back[0, :32]).all() and (back[0, 32:] == 1).all() and np.isnan(back[1, 32:]).all()


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("keys", [True, False])
def test_tiles_hold_every_code_once(fmt, dh, keys):
    at, scale_at = OP.places(fmt, dh, keys)
    assert sorted(at.ravel()) == list(range(64 * dh))
    n = 64 * dh * OP.FORMATS[fmt]["bits"] // 8
    assert sorted(scale_at.ravel()) == list(range(n, OP.tile_bytes(fmt, dh)))
    rng = np.random.default_rng(1)
    code, scale = rng.integers(0, 1 << OP.FORMATS[fmt]["bits"], (2, 128, dh), dtype=np.uint8), rng.integers(0, 256, (2, 128, dh // 32), dtype=np.uint8)
    tiles = OP.to_tiles(code, scale, fmt, keys)
    assert tiles.shape == (2, 2, OP.tile_bytes(fmt, dh))
    c, s = OP.from_tiles(tiles, fmt, dh, keys)
    assert np.array_equal(c, code) and np.array_equal(s, scale)
    # a row's bytes are its own: another row's codes do not touch them
    code[:, 5] = 0
    other = OP.to_tiles(code, scale, fmt, keys)
    c, _ = OP.from_tiles(other, fmt, dh, keys)
    assert (other != tiles).any() and np.array_equal(np.delete(c, 5, 1), np.delete(OP.from_tiles(tiles, fmt, dh, keys)[0], 5, 1))


def test_binding_refuses_tensors_that_do_not_fit():
    t = torch.zeros(1, 1, 1, 2176, dtype=torch.uint8)
    with pytest.raises(ValueError):
        mulo.make_packed_kv(t, t, 0, 64)          # not on a device
    with pytest.raises(ValueError):
        mulo.make_packed_kv(t, t, 5, 64)
    with pytest.raises(ValueError):
        mulo.make_kv_rows(None, None, 0)
    with pytest.raises(ValueError):
        mulo.make_kv_rows(torch.zeros(1, 1, 1, 64), torch.zeros(1, 1, 2, 64), 0)


@pytest.mark.parametrize("apart", [-HEAD + 16, -16, 16, HEAD - 16])
def test_keys_and_values_on_top_of_each_other_are_not_written(lib, apart):
    kv, r = split(dict(pv=(1 << 20) + apart))
    assert lib.mulo_pack_rows(None, C.byref(kv), C.byref(r)) == SHAPE
    for there in ("k", "v"):      # the one that the call leaves alone may lie anywhere
        kv, r = split({there: None, "pv": (1 << 20) + apart})
        assert lib.mulo_check_packed_rows(C.byref(kv), C.byref(r)) == 0
    # keys and values of a head in turn
    kv, r = split(dict(pv=(1 << 20) + HEAD, head=2 * HEAD, batch=4 * HEAD))
    assert lib.mulo_check_packed_rows(C.byref(kv), C.byref(r)) == 0


FAR = (1 << 40) - 8      # 2^24 rows of such a stride span 2^64 numbers


@pytest.mark.parametrize("changes", [dict(k_row=FAR, k_batch=1 << 40, v=None, pv=None), dict(v_row=FAR, v_batch=1 << 40, k=None, pk=None)], ids=["k", "v"])
def test_rows_on_top_of_each_other_whose_span_passes_64_bits(lib, changes):
    kv, r = split(dict(changes, rows=1 << 24, L=1 << 24, P=0, B=2, n_kv_heads=1, batch=1 << 30))
    assert lib.mulo_check_packed_rows(C.byref(kv), C.byref(r)) == 0
    assert lib.mulo_unpack_rows(None, C.byref(kv), C.byref(r)) == SHAPE


def test_outputs_on_top_of_each_other_whose_span_passes_64_bits(lib):
    a = attention_args(rows=1 << 24, L=1 << 24, P=0, B=2, n_kv_heads=1, n_heads=1, out_row=FAR, out_batch=1 << 40)
    assert lib.mulo_check_packed_attention(C.byref(a)) == SHAPE


# ---- keys and values on top of each other ----------------------------------------------------------------------------
PACK, UNPACK = 1, 2


def refusal(lib, writes, **changes):
    kv, r = split(changes)
    return lib.mulo_internal_check_rows(C.byref(kv), C.byref(r), writes)


@pytest.mark.parametrize("status, apart, changes", [
    (SHAPE, HEAD, {}), (SHAPE, -HEAD, {}), (SHAPE, 2 * HEAD, {}), (SHAPE, 7 * HEAD, {}), (SHAPE, -7 * HEAD + 16, {}), (SHAPE, 8 * HEAD - 16, {}), (0, 8 * HEAD, {}), (0, -8 * HEAD, {}),
    # a head, or a sequence, in turn
    (0, HEAD, dict(head=2 * HEAD, batch=4 * HEAD)), (SHAPE, 2 * HEAD, dict(head=2 * HEAD, batch=4 * HEAD)), (0, 3 * HEAD, dict(head=2 * HEAD, batch=4 * HEAD)),
    (0, 2 * HEAD, dict(batch=4 * HEAD)), (SHAPE, 3 * HEAD, dict(batch=4 * HEAD)), (0, 6 * HEAD, dict(batch=4 * HEAD)), (SHAPE, 12 * HEAD, dict(batch=4 * HEAD)), (0, 14 * HEAD, dict(batch=4 * HEAD)),
    # gaps of exactly a head
    (0, HEAD, dict(head=3 * HEAD, batch=6 * HEAD)), (0, 2 * HEAD, dict(head=3 * HEAD, batch=6 * HEAD)), (SHAPE, 2 * HEAD + 16, dict(head=3 * HEAD, batch=6 * HEAD)),
    # heads outside of sequences
    (SHAPE, 4 * HEAD, dict(batch=HEAD, head=4 * HEAD)), (0, 8 * HEAD, dict(batch=HEAD, head=4 * HEAD)),
], ids=str)
def test_keys_on_values_of_another_head_are_not_written(lib, status, apart, changes):
    assert refusal(lib, PACK, pv=(1 << 20) + apart, **changes) == status
    if status:
        kv, r = split(dict(changes, pv=(1 << 20) + apart))
        assert lib.mulo_pack_rows(None, C.byref(kv), C.byref(r)) == status
    assert refusal(lib, UNPACK, pv=(1 << 20) + apart, v=1 << 18, **changes) == 0       # read only


# rows of numbers, bytes from the keys to the values: 3 rows of 64 bf16 numbers of 2 heads of 4 sequences are 3072 bytes
TOKENS = dict(k_row=128, k_head=64, k_batch=384, v_row=128, v_head=64, v_batch=384)
FUSED = dict(k_row=256, k_head=64, k_batch=768, v_row=256, v_head=64, v_batch=768)      # a token's keys, then its values


@pytest.mark.parametrize("status, apart, changes", [
    (SHAPE, 16, {}), (SHAPE, -16, {}), (SHAPE, 768, {}), (SHAPE, 3056, {}), (0, 3072, {}), (0, -3072, {}), (SHAPE, 3072, dict(dtype=0)), (0, 6144, dict(dtype=0)),
    (SHAPE, 256, TOKENS), (SHAPE, 128, TOKENS), (0, 3072, TOKENS),
    (0, 256, FUSED), (0, -256, FUSED), (SHAPE, 128, FUSED), (SHAPE, 240, FUSED), (0, 512 + 256, FUSED), (SHAPE, 512, FUSED), (0, 1536 + 256, FUSED),
    # heads of keys and, behind them, channels of rows; of other steps inside a head
    (0, 384, dict(ACROSS, k_head=384, v_head=384, k_batch=768, v_batch=768)), (SHAPE, 382, dict(ACROSS, k_head=384, v_head=384, k_batch=768, v_batch=768)),
    (SHAPE, 384, dict(ACROSS, v_chan=4, k_head=384, v_head=384, k_batch=768, v_batch=768)),
    # values in the gaps of every second row of the keys, and on one of their rows
    (0, 128, dict(k_row=128, k_head=1024, k_batch=4096, v_row=256, v_head=1024, v_batch=4096)), (SHAPE, 128 + 64, dict(k_row=128, k_head=1024, k_batch=4096, v_row=192, v_head=1024, v_batch=4096)),
    # batches of other steps far apart
    (0, 1 << 30, dict(v_batch=1 << 20)),
], ids=str)
def test_rows_on_top_of_each_other_are_not_written(lib, status, apart, changes):
    assert refusal(lib, UNPACK, k=1 << 20, v=(1 << 20) + apart, pv=1 << 25, **changes) == status
    if status:
        kv, r = split(dict(changes, k=1 << 20, v=(1 << 20) + apart))
        assert lib.mulo_unpack_rows(None, C.byref(kv), C.byref(r)) == status
    assert refusal(lib, PACK, k=1 << 20, v=(1 << 20) + apart, pv=1 << 25, **changes) == 0       # read only


def test_steps_that_interleave_without_end(lib):
    """Keys every 128 numbers, values of unlike steps in their gaps: gone through up to a limit."""
    far = dict(B=1, n_kv_heads=1, rows=1 << 20, P=0, k=1 << 20, v=(1 << 20) + 128, pv=1 << 40, k_row=128, v_row=256, batch=0, head=0)
    assert refusal(lib, UNPACK, L=1000, **far) == 0
    assert refusal(lib, UNPACK, L=1 << 18, **far) == UNSUPPORTED


def test_random_layouts_against_sets_of_places(lib):
    rng = np.random.default_rng(5)

    def places(dims, run):
        at = np.arange(run)
        for n, step in dims:
            at = (at[None] + (np.arange(n) * step).reshape(-1, *[1] * at.ndim)).reshape(-1)
        return at

    def nested(dims, unit, tight):
        """Steps that step over what lies inside, the dimensions in a random order of nesting."""
        steps, extent = [0] * len(dims), unit[1]
        for i in rng.permutation(len(dims)):
            steps[i] = -(-extent // unit[0]) * unit[0] + unit[0] * int(rng.integers(0, 1 if tight else 20))
            extent += (dims[i] - 1) * steps[i]
        return steps

    found = {0: 0, SHAPE: 0}
    for trial in range(1500):
        B, nkv, L = (int(x) for x in rng.integers(1, 4, 3))
        across, alike = trial % 3 == 0, trial % 2
        ks = nested([B, nkv, L], (8, 64), rng.random() < 0.3)
        if across:
            extent = L + int(rng.integers(1, 9))      # (1: rows of channels)
            outer = nested([B, nkv], (1, 63 * extent + L), rng.random() < 0.3)
            if alike:      # steps that step over the keys and the values of a head
                inside = max(63 * extent + L, 64 + (L - 1) * ks[2]) + 64 * int(rng.integers(0, 60))
                outer = nested([B, nkv], (8, inside), True)
                ks[:2] = outer
            vs, chan = outer + [1], extent
        else:
            vs, chan = list(ks) if alike else nested([B, nkv, L], (8, 64), rng.random() < 0.3), 1
        kp, vp = places(list(zip((B, nkv, L), ks)), 64), places(list(zip((B, nkv, L, 64), vs + [chan])), 1)
        if len(set(kp)) < len(kp) or len(set(vp)) < len(vp):
            continue
        off = int(rng.integers(-(vp.max() + 20), kp.max() + 20)) if rng.random() < 0.5 else int(rng.choice(ks)) + 64 * int(rng.integers(-2, 3))
        if not across or chan == 1:
            off = off // 8 * 8
        want = SHAPE if np.intersect1d(kp, vp + off).size else 0
        got = refusal(lib, UNPACK, B=B, n_kv_heads=nkv, L=L, P=0, k=1 << 20, v=(1 << 20) + 2 * off, batch=1 << 20, head=1 << 16, pv=1 << 30,
                      k_batch=ks[0], k_head=ks[1], k_row=ks[2], v_batch=vs[0], v_head=vs[1], v_row=vs[2], v_chan=chan)
        assert got == want, (B, nkv, L, ks, vs, chan, off)
        found[want] += 1
        # a cache of the same arrangement, in tiles
        hs = nested([B, nkv], (16, HEAD), rng.random() < 0.3)
        cp = places(list(zip((B, nkv), hs)), HEAD)
        off = int(rng.integers(-(cp.max() + 64), cp.max() + 64)) // 16 * 16 if rng.random() < 0.5 else HEAD * int(rng.integers(1, 9)) + 16 * int(rng.integers(-1, 2))
        want = SHAPE if np.intersect1d(cp[::16], cp[::16] + off).size else 0
        assert refusal(lib, PACK, B=B, n_kv_heads=nkv, batch=hs[0], head=hs[1], pk=1 << 25, pv=(1 << 25) + off) == want, (B, nkv, hs, off)
        found[want] += 1
    assert min(found.values()) > 300, found


@pytest.mark.parametrize("how", ["rows", "whole", "odd"])
@pytest.mark.parametrize("L", [1, 3, 8])
def test_a_number_written_beside_the_rows_is_noticed(how, L):
    """The check that the tests on the card use: every place of the buffer but the rows' own."""
    from tests.test_gpu_packed import inside, outside_is_seven
    w, view = inside((2, 2, L, 4), how, torch.float32, "cpu")
    view.fill_(1.0)
    flat, own = w.view(-1), (w == 1).view(-1).clone()
    assert own.sum() == view.numel() and not own[0] and not own[-1] and outside_is_seven(w, view)
    for i in range(w.numel()):
        if not own[i]:
            flat[i] = 1.0
            assert not outside_is_seven(w, view), i
            flat[i] = 7.0
