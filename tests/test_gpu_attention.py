"""mulo_attention through the C ABI against its definition in float64 (oracle/context.py), over types, head layouts, lengths,
windows, ragged and absent sequences, strides and memory that nothing may read."""
import pytest
import torch

import paper_2601_05149_amd as mulo
from oracle import context as OC
from tests.gpu_util import DEV, say

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN = float("nan")


def sees(p, L, n, sinks, window):
    """[L, n]: which of n positions the queries at p, p + 1, ... see."""
    t, at = torch.arange(n), torch.arange(p, p + L)[:, None]
    return (t <= at) & (torch.tensor(window == 0) | (t < sinks) | (at - t < window))


def make(dtype, B, L, nh, nkv, dh, P, G=1, S=0, sinks=0, window=0, starts=None, seed=0, gain=1.0, rows=None):
    g = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    normal = lambda *shape: torch.randn(*shape, generator=g).to(dt)
    rows = (P + L + 7) // 8 * 8 if rows is None else rows
    srows = (S + 7) // 8 * 8
    c = dict(q=normal(B, nh, L, dh).mul(gain), k=normal(B, nkv, rows, dh), v=normal(B, nkv, dh, rows), P=P, S=S, sinks=sinks, window=window,
             starts=[P] * B if starts is None else starts, pk=normal(G, nkv, srows, dh) if S else None,
             pv=normal(G, nkv, dh, srows) if S else None, ragged=starts is not None, bf16=dtype == "bf16")
    # rows that no query of the call sees hold NaN
    own, pre = torch.zeros(B, rows, dtype=torch.bool), torch.zeros(G, max(srows, 1), dtype=torch.bool)
    c["starts"] = [min(p, rows - L) for p in c["starts"]]
    for b, p in enumerate(c["starts"]):
        if p >= 0:
            seen = sees(S + p, L, S + p + L, sinks, window).any(0)
            pre[b // (B // G), :S] |= seen[:S]
            own[b, :p + L] |= seen[S:]
    for b in range(B):
        c["k"][b, :, ~own[b]] = NAN
        c["v"][b, :, :, ~own[b]] = NAN
    for i in range(G if S else 0):
        c["pk"][i, :, ~pre[i]] = NAN
        c["pv"][i, :, :, ~pre[i]] = NAN
    return c


def plan_of(c, d, out, **kw):
    P_seq = torch.tensor(c["starts"], dtype=torch.int32, device=DEV) if c["ragged"] else None
    return mulo.make_attention(d["q"], out, d["k"], d["v"], c["P"], P_seq=P_seq, prefix_k=d["pk"], prefix_v=d["pv"], prefix_len=c["S"],
                               sinks=c["sinks"], window=c["window"], **kw)


def on_device(c):
    return {n: None if c[n] is None else c[n].to(DEV) for n in ("q", "k", "v", "pk", "pv")}


def workspace(plan, fill=0xFF):
    n = mulo.mulo_attention_workspace_bytes(plan)
    return torch.full((n,), fill, dtype=torch.uint8, device=DEV) if n else None      # 0xFF..: NaN as bf16 and as float32


def plain(c):
    """The definition with the queries of a sequence side by side, for cases that the oracle takes too long over; float64, on the device."""
    B, nh, L, dh = c["q"].shape
    group, S = nh // c["k"].shape[1], c["S"]
    out, mass = torch.zeros(B, nh, L, dh, dtype=torch.float64), torch.zeros(B, nh, L, dh, dtype=torch.float64)
    reach, keys = torch.zeros(B, nh, L, dtype=torch.float64), torch.zeros(B, L)
    for b, p in enumerate(c["starts"]):
        if p < 0:
            continue
        n = S + p + L
        K, V = c["k"][b, :, :p + L], c["v"][b, :, :, :p + L].transpose(1, 2)
        if S:
            g = b // (B // c["pk"].shape[0])
            K, V = torch.cat([c["pk"][g, :, :S], K], 1), torch.cat([c["pv"][g, :, :, :S].transpose(1, 2), V], 1)
        see = sees(S + p, L, n, c["sinks"], c["window"])
        keys[b] = see.sum(1)
        see = see.to(DEV)
        for h in range(nh):
            q, Kh, Vh = c["q"][b, h].to(DEV).double(), K[h // group].to(DEV).double(), V[h // group].to(DEV).double()
            Kh, Vh = torch.nan_to_num(Kh), torch.nan_to_num(Vh)          # no query sees those rows
            z = (q @ Kh.t().contiguous() * dh ** -0.5).masked_fill(~see, float("-inf"))
            e = torch.exp(z - z.max(-1, keepdim=True).values)
            w = e / e.sum(-1, keepdim=True)
            out[b, h], mass[b, h] = (w @ Vh).cpu(), (w @ Vh.abs()).cpu()
            reach[b, h] = (q.abs() @ Kh.abs().t().contiguous() * dh ** -0.5).masked_fill(~see, 0.0).max(-1).values.cpu()
    return out, mass, reach, keys


def check(c, out, label, scale=None, reference=None):
    # a NaN in the caches would spread through the oracle's products, which take the visible rows only
    want, mass, reach, keys = reference or OC.context_attention(c["q"], c["k"], c["v"], c["starts"], c["pk"], c["pv"], c["S"], c["sinks"], c["window"], scale)
    tol = OC.tolerance(mass, reach, keys, want, c["q"].shape[-1], c["bf16"])
    err = (out.double().cpu() - want).abs()
    assert torch.isfinite(out).all(), "%s: not finite" % label
    worst = (err / (tol + 1e-30)).max().item()
    say("  %s: worst error %.3g of the bound" % (label, worst))
    assert (err <= tol).all(), "%s: %.3g of the bound" % (label, worst)


CASES = [
    # one key; a key of the prefix and its own; the ends of a tile of keys
    ("bf16", 1, 1, 1, 1, 64, 0, {}),
    ("f32", 1, 1, 1, 1, 128, 0, dict(S=1)),
    ("bf16", 2, 1, 2, 2, 128, 63, dict(S=64)),
    ("bf16", 2, 1, 2, 2, 128, 64, dict(S=65)),
    ("f32", 2, 2, 2, 2, 64, 30, dict(S=31)),
    ("f32", 3, 1, 2, 1, 128, 127, dict(S=129)),
    # many single tokens behind one prefix, and behind two (guidance)
    ("bf16", 33, 1, 2, 2, 128, 100, dict(S=333)),
    ("bf16", 64, 1, 2, 2, 64, 70, dict(S=500, G=2)),
    ("f32", 24, 1, 2, 2, 128, 70, dict(S=200, G=2)),
    # more stacked rows than a workgroup takes, with and without shared key heads
    ("bf16", 48, 4, 2, 2, 64, 37, dict(S=150)),
    ("bf16", 20, 5, 8, 2, 128, 90, dict(S=77)),
    ("f32", 20, 3, 8, 2, 64, 90, dict(S=77, G=4)),
    # blocks: a few rows, ragged tiles of queries, shared key heads, one group per sequence
    ("bf16", 2, 33, 4, 4, 128, 50, dict(S=40)),
    ("bf16", 3, 130, 4, 1, 64, 11, dict(S=100)),
    ("bf16", 2, 300, 2, 2, 128, 5, dict(S=70, G=2)),
    ("f32", 2, 150, 4, 2, 128, 9, dict(S=33)),
    ("f32", 1, 260, 2, 2, 64, 0, {}),
    ("bf16", 1, 257, 2, 2, 64, 0, {}),
    # blocks whose keys are dealt to several workgroups
    ("bf16", 1, 150, 4, 2, 128, 900, dict(S=100)),
    ("f32", 1, 140, 2, 2, 128, 300, {}),
    ("bf16", 2, 135, 2, 2, 64, 1000, dict(window=900, sinks=30, starts=[1000, -1])),
    ("f32", 2, 133, 2, 1, 64, 200, dict(S=70, starts=[50, 200])),
    # windows: one key, shorter than a tile, longer than everything, across the border of prefix and own rows, sinks in both
    ("bf16", 2, 1, 2, 2, 128, 200, dict(window=1)),
    ("f32", 2, 7, 2, 2, 64, 200, dict(window=1, sinks=1)),
    ("bf16", 3, 5, 4, 2, 128, 300, dict(window=17, sinks=4)),
    ("bf16", 2, 1, 2, 2, 64, 3000, dict(window=200, sinks=5)),
    ("bf16", 2, 40, 2, 2, 64, 100, dict(window=1000, sinks=3)),
    ("bf16", 4, 3, 2, 2, 128, 20, dict(S=300, window=100, sinks=70)),
    ("bf16", 6, 1, 2, 2, 128, 500, dict(S=300, window=100, sinks=20)),
    ("f32", 4, 3, 2, 2, 128, 20, dict(S=100, window=40, sinks=130, G=2)),
    ("bf16", 4, 9, 4, 4, 64, 400, dict(S=100, window=64, sinks=230)),
    ("bf16", 2, 290, 2, 2, 128, 400, dict(window=130, sinks=10)),
    ("bf16", 2, 290, 4, 2, 64, 100, dict(S=200, window=150, sinks=30)),
    ("f32", 1, 200, 2, 2, 64, 300, dict(window=90, sinks=70)),
    # a window and sinks as large as they come
    ("bf16", 2, 3, 2, 2, 128, 70, dict(S=40, window=2 ** 31 - 1, sinks=2 ** 31 - 1)),
    ("f32", 1, 140, 2, 2, 64, 70, dict(window=2 ** 31 - 1)),
    ("bf16", 2, 1, 2, 2, 64, 700, dict(S=40, window=30, sinks=2 ** 31 - 1)),
    # a window that never reaches the prefix, without sinks: the prefix is not read at all
    ("bf16", 4, 2, 2, 2, 128, 300, dict(S=64, window=50)),
    # sequences of unequal length, absent ones, one that is longer than the cache allows
    ("bf16", 5, 1, 2, 2, 128, 200, dict(S=90, starts=[200, 0, -1, 77, 10000])),
    ("bf16", 4, 6, 4, 2, 64, 200, dict(S=90, G=2, starts=[-1, -5, 200, 3], window=60, sinks=7)),
    ("f32", 4, 1, 2, 2, 64, 200, dict(S=33, starts=[-1, 200, 64, 63])),
    ("bf16", 3, 140, 2, 2, 128, 100, dict(starts=[-1, 100, 0])),
    ("bf16", 3, 140, 2, 2, 64, 300, dict(starts=[300, 250, 0], window=77, sinks=3)),
    ("bf16", 2, 1, 2, 2, 128, 50, dict(S=20, starts=[-1, -1])),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%dx%d-h%d.%d-%d-P%d%s" % (c[:7] + ("".join("-%s%s" % (k, v) for k, v in c[7].items() if k != "starts"),)))
def test_attention(case):
    dtype, B, L, nh, nkv, dh, P, kw = case
    c = make(dtype, B, L, nh, nkv, dh, P, **kw)
    d = on_device(c)
    for use in (True, False):            # with the scratch it asks for (holding NaN), and with none
        out = torch.full_like(d["q"], NAN)
        plan = plan_of(c, d, out)
        mulo.mulo_attention(plan, workspace(plan) if use else None)
        torch.cuda.synchronize()
        check(c, out, "scratch" if use else "no scratch")


# Sizes at which keys are dealt to several workgroups, and those of more queries
DEALT = [
    # the rows of all sequences over the prefix together: single tokens, two and three groups, shared key heads, more than 64 rows of a
    # sequence, ragged and absent sequences, a window that cuts the prefix, sinks that the window has left behind
    ("bf16", 8, 1, 8, 8, 128, 70, dict(S=1000)),
    ("bf16", 10, 1, 8, 8, 64, 100, dict(S=1801, G=2)),
    ("bf16", 15, 5, 16, 4, 128, 150, dict(S=1901, G=3)),
    ("bf16", 16, 24, 8, 4, 64, 30, dict(S=4000)),
    ("bf16", 16, 91, 8, 8, 64, 9, dict(S=3001)),
    ("bf16", 8, 3, 8, 8, 128, 300, dict(S=1000, starts=[300, 0, -1, 5, 64, 63, 128, -9])),
    ("bf16", 8, 2, 8, 8, 128, 200, dict(S=1500, window=1300, sinks=130)),
    ("bf16", 8, 2, 8, 8, 128, 400, dict(S=1500, window=300, sinks=1400)),
    ("f32", 16, 3, 8, 8, 64, 40, dict(S=333)),
    ("f32", 8, 7, 8, 4, 128, 100, dict(S=500, G=2, starts=[-1, 100, 0, 31, 32, 33, -1, 99])),
    ("f32", 8, 40, 8, 8, 64, 70, dict(S=400)),
    # each sequence on its own, its keys dealt to 8 and more workgroups
    ("bf16", 2, 1, 4, 4, 128, 1500, {}),
    ("bf16", 1, 100, 2, 2, 128, 1700, {}),
    ("bf16", 3, 16, 8, 1, 64, 1600, dict(window=1555, sinks=33)),
    ("bf16", 3, 4, 4, 2, 128, 1800, dict(starts=[1800, -1, 3], window=1700, sinks=2)),
    ("bf16", 2, 1, 4, 2, 128, 900, dict(S=800, G=2, starts=[10, 900])),
    ("bf16", 16, 45, 8, 4, 128, 30, dict(S=2500)),
    # float32 over few keys: a tile a wavefront
    ("f32", 3, 5, 4, 2, 128, 60, dict(S=33)),
    ("f32", 2, 40, 2, 2, 128, 300, dict(window=20, sinks=3)),
    ("f32", 4, 2, 4, 2, 128, 50, dict(S=20, G=2, starts=[50, -1, 0, 7])),
    ("f32", 3, 70, 2, 1, 64, 100, dict(S=40, starts=[-1, 100, 31], window=90, sinks=41)),
    # long blocks: 256 and 128 queries a workgroup over tiles of 128 keys
    ("bf16", 5, 150, 32, 32, 128, 33, dict(S=77)),
    ("bf16", 4, 150, 32, 32, 128, 33, {}),
    ("bf16", 5, 140, 32, 8, 128, 100, dict(starts=[100, -1, 0, 17, 64], S=50)),
    ("bf16", 5, 260, 32, 32, 128, 60, dict(window=100, sinks=10)),
    ("bf16", 8, 150, 32, 32, 64, 40, dict(S=200, window=150, sinks=9)),
    ("f32", 2, 150, 2, 2, 64, 900, dict(S=70)),
]
name_of = lambda c: "%s-%dx%d-h%d.%d-%d-P%d%s" % (c[:7] + ("".join("-%s%s" % (k, v) for k, v in c[7].items() if k != "starts"),))


@pytest.mark.parametrize("case", [CASES[i] for i in (2, 11, 20, 29, 40)], ids=name_of)
def test_plain_form_is_the_oracle(case):
    dtype, B, L, nh, nkv, dh, P, kw = case
    c = make(dtype, B, L, nh, nkv, dh, P, **kw)
    out, mass, reach, keys = plain(c)
    want = OC.context_attention(c["q"], c["k"], c["v"], c["starts"], c["pk"], c["pv"], c["S"], c["sinks"], c["window"])
    # Two forms of float64, each off by what the bound of the oracle's module says of float32 with 2^-53 for 2^-24 (and 2^-50 for an
    # exponential's 2^-22): a score by (dh + 8) 2^-53 reach, so a weight, numerator and denominator, by twice that; sums of n terms
    # by (n + 8) 2^-53, twice.
    rel = 2 * ((dh + 8) * 2.0 ** -53 * reach + 2.0 ** -50) + 2 * (keys[:, None, :] + 8) * 2.0 ** -53
    far = [((a - b).abs() > 2 * tol).sum().item() for a, b, tol in zip(
        (out, mass, reach), want, (mass * rel[..., None], mass * rel[..., None], (dh + 8) * 2.0 ** -53 * reach))]
    assert far == [0, 0, 0] and torch.equal(keys, want[3])


@pytest.mark.parametrize("case", DEALT, ids=name_of)
def test_dealt_keys_and_many_queries(case):
    dtype, B, L, nh, nkv, dh, P, kw = case
    c = make(dtype, B, L, nh, nkv, dh, P, **kw)
    d = on_device(c)
    reference = plain(c)
    plan = plan_of(c, d, torch.empty_like(d["q"]))
    asked = mulo.mulo_attention_workspace_bytes(plan)
    least = B * nh * L * (dh + 2) * 4
    for share in (1.0, 0.6, 0.0):            # with the scratch it asks for (holding NaN), with less, and with none
        out = torch.full_like(d["q"], NAN)
        n = int(asked * share) // 4 * 4
        mulo.mulo_attention(plan_of(c, d, out), torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) if n else None)
        torch.cuda.synchronize()
        check(c, out, "%d of %d results of a query" % (n // least, asked // least), reference=reference)


ABSENT = [c for c in CASES + DEALT if any(p < 0 for p in c[7].get("starts", ()))] + [
    # every row over the prefix together: 16 sequences, half of them absent
    ("bf16", 16, 2, 8, 8, 64, 100, dict(S=4000, starts=[100, -1] * 8)),
]


@pytest.mark.parametrize("case", ABSENT, ids=name_of)
def test_absent_sequences_are_zeros_whatever_their_queries_hold(case):
    """A slot without a sequence may hold infinities, NaN, or numbers whose scores overflow: its outputs are zeros, and those of the
    other sequences have the bits they have beside a slot of ordinary numbers."""
    dtype, B, L, nh, nkv, dh, P, kw = case
    c = make(dtype, B, L, nh, nkv, dh, P, **kw)
    d = on_device(c)
    absent = torch.tensor([p < 0 for p in c["starts"]])
    ask = mulo.mulo_attention_workspace_bytes(plan_of(c, d, torch.empty_like(d["q"])))
    for share in (1.0, 0.0):
        ws = torch.full((int(ask * share),), 0xFF, dtype=torch.uint8, device=DEV) if int(ask * share) else None
        want = torch.full_like(d["q"], NAN)
        mulo.mulo_attention(plan_of(c, d, want), ws)
        for bad in (float("inf"), float("-inf"), NAN, torch.finfo(DT[dtype]).max):
            q = d["q"].clone()
            q[absent.to(DEV)] = bad
            out = torch.full_like(q, NAN)
            mulo.mulo_attention(plan_of(c, dict(d, q=q), out), ws)
            torch.cuda.synchronize()
            assert (out[absent.to(DEV)] == 0).all(), "queries of %s, scratch %s" % (bad, ws is not None)
            assert torch.equal(out, want), "queries of %s, scratch %s" % (bad, ws is not None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sharp_and_scaled_scores(dtype):
    """Scores of a hundred and more: nearly all of the mass on one key; and a scale of the caller's."""
    c = make(dtype, 3, 4, 4, 2, 128, 150, S=70, gain=12.0)
    d = on_device(c)
    for scale in (None, 0.25):
        out = torch.full_like(d["q"], NAN)
        plan = plan_of(c, d, out, scale=scale or 0.0)
        mulo.mulo_attention(plan, workspace(plan))
        torch.cuda.synchronize()
        check(c, out, "scale %s" % scale, scale)


@pytest.mark.parametrize("L", [1, 150])
def test_strides(L):
    """Token-major queries and output inside a wider row, keys that are interleaved over heads, values of heads in front of
    sequences; what lies around the output stays as it was."""
    B, nh, nkv, dh, P, S = 3, 4, 2, 64, 40, 50
    c = make("bf16", B, L, nh, nkv, dh, P, S=S)
    d = on_device(c)
    rows = d["k"].shape[2]
    wide = torch.full((B, L, nh + 2, dh), 7.0, dtype=torch.bfloat16, device=DEV)
    out = wide[:, :, 1:nh + 1].permute(0, 2, 1, 3)
    qs = torch.zeros(B, L, nh, 2 * dh, dtype=torch.bfloat16, device=DEV)
    qs[..., :dh] = d["q"].permute(0, 2, 1, 3)
    d["q"] = qs[..., :dh].permute(0, 2, 1, 3)
    d["k"] = d["k"].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    v = torch.full((nkv, B, dh, rows + 24), NAN, dtype=torch.bfloat16, device=DEV)
    v[..., 8:8 + rows] = d["v"].transpose(0, 1)
    d["v"] = v[..., 8:8 + rows].transpose(0, 1)
    d["pk"] = d["pk"].transpose(1, 2).contiguous().transpose(1, 2)
    plan = plan_of(c, d, out)
    mulo.mulo_attention(plan, workspace(plan))
    torch.cuda.synchronize()
    check(c, out, "strided")
    assert (wide[:, :, 0] == 7).all() and (wide[:, :, nh + 1] == 7).all()


def test_offsets_beyond_32_bits():
    """The last rows of a cache whose head is longer than 2^32 bytes: the same as those rows on their own."""
    rows, n, dh = (1 << 24) + 0, 304, 128
    g = torch.Generator().manual_seed(3)
    normal = lambda *s: torch.randn(*s, generator=g).bfloat16().to(DEV)
    k, v = torch.empty(1, 1, rows, dh, dtype=torch.bfloat16, device=DEV), torch.empty(1, 1, dh, rows, dtype=torch.bfloat16, device=DEV)
    k[:, :, rows - n:], v[..., rows - n:] = normal(1, 1, n, dh), normal(1, 1, dh, n)
    k[:, :, :8], v[..., :8] = normal(1, 1, 8, dh), normal(1, 1, dh, 8)
    for L in (1, 140):
        q = normal(1, 2, L, dh)
        outs = []
        for kk, vv, P in ((k, v, rows - L), (torch.cat([k[:, :, :8], k[:, :, rows - n:]], 2), torch.cat([v[..., :8], v[..., rows - n:]], 3), n + 8 - L)):
            out = torch.empty_like(q)
            plan = mulo.make_attention(q, out, kk, vv, P, sinks=8, window=150)
            mulo.mulo_attention(plan, workspace(plan))
            outs.append(out)
        torch.cuda.synchronize()
        off = (outs[0].float() - outs[1].float()).abs().max().item()
        assert torch.isfinite(outs[0]).all() and off <= 2.0 ** -6, off      # keys meet in other tiles: other roundings


@pytest.mark.parametrize("dtype, nh, S", [("bf16", 4, 300), ("bf16", 8, 1300), ("f32", 4, 300)])
def test_bits_do_not_depend_on_the_workspace_or_the_run(dtype, nh, S):
    c = make(dtype, 8, 1, nh, nh, 128, 500, S=S, G=2)
    d = on_device(c)
    outs = []
    for fill in (0, 0xFF, 0x7F):
        out = torch.full_like(d["q"], NAN)
        plan = plan_of(c, d, out)
        mulo.mulo_attention(plan, workspace(plan, fill))
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("nh, S", [(4, 90), (16, 1801)])
def test_recorded_and_replayed_with_growing_sequences(nh, S):
    """One graph serves a decoding loop: the lengths live on the device, the launch is sized by the longest."""
    c = make("bf16", 6, 1, nh, nh, 64, 300, S=S, starts=[300] * 6)
    for t in ("k", "v", "pk", "pv"):
        c[t] = torch.nan_to_num(c[t])
    d = on_device(c)
    side = torch.cuda.Stream()
    P_seq = torch.zeros(6, dtype=torch.int32, device=DEV)
    out = torch.empty_like(d["q"])
    plan = mulo.make_attention(d["q"], out, d["k"], d["v"], 300, P_seq=P_seq, prefix_k=d["pk"], prefix_v=d["pv"], prefix_len=S)
    ws, other = workspace(plan), torch.empty_like(out)
    with torch.cuda.stream(side):
        mulo.mulo_attention(plan, ws)
        side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        mulo.mulo_attention(plan, ws)
    with torch.cuda.stream(side):
        for rep, lens in enumerate(([0, 1, 2, 63, 64, 65], [300, 299, -1, 5, 100, 0], [7] * 6, [300] * 6)):
            P_seq.copy_(torch.tensor(lens, dtype=torch.int32))
            out.fill_(NAN)
            graph.replay()
            side.synchronize()
            c["starts"] = lens
            check(c, out, "replay %d" % rep)
            eager = mulo.make_attention(d["q"], other, d["k"], d["v"], 300, P_seq=P_seq, prefix_k=d["pk"], prefix_v=d["pv"], prefix_len=S)
            mulo.mulo_attention(eager, workspace(eager))
            side.synchronize()
            assert torch.equal(out, other)
    del graph
