"""mulo_sample_filtered through the C ABI against its definition in float64 (oracle/sampling.py)."""
import itertools

import numpy as np
import pytest
import torch

import paper_2601_05149_amd as mulo
from oracle import sampling as OS
from tests.gpu_util import DEV, say

pytestmark = pytest.mark.gpu
INF = float("inf")


def run(z, u, in_place=False, **kw):
    """tokens, probs, logits of one call on z (a device tensor, any row stride)."""
    p = mulo.make_sample_params(**kw)
    R = z.shape[0] // 2 if kw.get("cfg_scale") else z.shape[0]
    V = z.shape[1]
    tokens = torch.full((R,), -7, dtype=torch.int32, device=DEV)
    probs = torch.full((R, V), 9.0, device=DEV)
    out = z[:R] if in_place else torch.full((R, V), 9.0, device=DEV)
    mulo.mulo_sample_filtered(p, z, u, tokens, probs, out)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), probs.cpu().numpy(), out.cpu().numpy()


def check(z, u, **kw):
    cfg = kw.get("cfg_scale", 0.0)
    rows = OS.row_logits(z.float().cpu().numpy(), cfg)
    tokens, probs, out = run(z, u, **kw)
    f = {k: v for k, v in kw.items() if k != "cfg_scale"}
    T = kw.get("temperature", 1.0)
    for r, row in enumerate(rows):
        w = OS.kept(row, **f)
        at = sorted(w)
        assert np.array_equal(np.nonzero(np.isfinite(out[r]))[0], at), "row %d: another set stays" % r
        # the quotient is rounded once, half a step of float32 (of its smallest numbers 2^-150), and kept finite
        most = float(np.finfo(np.float32).max)
        assert np.allclose(out[r][at], np.clip(row[at].astype(np.float64) / (T or 1.0), -most, most), rtol=2.0 ** -24, atol=2.0 ** -150)
        total = sum(w.values())
        want = np.zeros(len(row))
        for i in at:
            want[i] = w[i] / total
        # a weight is an integer multiple of 2^-44 of the largest one, half a step off; the result is rounded to float32
        assert np.all(np.abs(probs[r] - want) <= 2.0 ** -24 * want + 2.0 ** -44 + 1e-45), "row %d: probabilities" % r
        tok, far = OS.draw(w, float(u[r]))
        if tokens[r] != tok:                     # sums of up to 262144 weights, each half a step of 2^-44 off
            assert far < len(row) * 2.0 ** -45, "row %d: token %d, not %d (%.3g from a border)" % (r, tokens[r], tok, far)
    return tokens


def rows_of(R, V, seed=0, spread=1.5, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(R, V, generator=g) * spread).to(dtype).to(DEV), torch.rand(R, generator=g).to(DEV)


@pytest.mark.parametrize("V", [1, 2, 3, 5, 64, 255, 256, 257, 1000, 1024, 4097, 16384, 20001])
def test_vocabularies(V):
    z, u = rows_of(3, V, seed=V)
    check(z, u)
    check(z, u, temperature=0.7, top_k=max(1, V // 3), top_p=0.8, min_p=0.01)


@pytest.mark.parametrize("V", [1000, 4000, 16000, 20001])
def test_more_rows_than_compute_units(V):
    """Many rows are dealt otherwise than few: the first and last against the definition, all with the bits they have in small calls."""
    R = torch.cuda.get_device_properties(0).multi_processor_count + 9
    z, u = rows_of(R, V, seed=V)
    for kw in (dict(top_k=700, top_p=0.9), dict(temperature=0.8, top_p=0.9, min_p=1e-3), dict(top_k=60)):
        every = run(z, u, **kw)
        for a, b in ((0, 3), (R // 2, R // 2 + 100), (R - 3, R)):
            few = run(z[a:b], u[a:b].contiguous(), **kw)
            for x, y in zip(every, few):
                assert np.array_equal(x[a:b].view(np.int32), y.view(np.int32))
        check(z[-2:], u[-2:].contiguous(), **kw)


@pytest.mark.parametrize("dtype, cfg", [(torch.bfloat16, 0.0), (torch.float32, 3.0), (torch.bfloat16, 1.7)])
def test_large_vocabularies_of_every_kind(dtype, cfg):
    for V in (32769, 60001):
        z, u = rows_of(4, V, seed=V, spread=2.0, dtype=dtype)
        u = u[:2].contiguous() if cfg else u
        for kw in (dict(top_k=300, top_p=0.9), dict(temperature=0.7, top_p=0.95, min_p=1e-3), dict(top_k=5000), dict(temperature=0.0)):
            check(z, u, cfg_scale=cfg, **kw)


@pytest.mark.parametrize("V", [32765, 32768])
def test_the_longest_rows_that_are_kept_in_lds(V):
    """One row, and more rows than compute units, at the most LDS a workgroup takes."""
    z, u = rows_of(3, V, seed=V, spread=2.0)
    for kw in (dict(), dict(top_k=2048, top_p=0.9), dict(temperature=0.8, top_p=0.95, min_p=1e-3), dict(top_k=2049)):
        check(z, u, **kw)
    R = torch.cuda.get_device_properties(0).multi_processor_count + 3
    z, u = rows_of(R, V, seed=V + 1, spread=2.0)
    every = run(z, u, top_k=900, top_p=0.9)
    for a, b in ((0, 2), (R - 2, R)):
        for x, y in zip(every, run(z[a:b], u[a:b].contiguous(), top_k=900, top_p=0.9)):
            assert np.array_equal(x[a:b].view(np.int32), y.view(np.int32))


LONG = 40001       # a row that is read again in every pass


@pytest.mark.parametrize("dtype, cfg", [(torch.float32, 0.0), (torch.bfloat16, 0.0), (torch.float32, 2.0), (torch.bfloat16, 2.0)])
def test_long_rows_with_ties(dtype, cfg):
    """Some 10000 entries of each value, all of them alike, and zeros of both signs: borders inside a tie, with more entries than the
    list holds in front of them and with fewer."""
    g = torch.Generator().manual_seed(31)
    z = torch.randint(0, 4, (3, LONG), generator=g).float()
    z[1] = 0.0
    z[2, 100:] = -0.0
    z[2, :100] = 0.0
    if cfg:      # the guided row is z_u + 2 (z_c - z_u): of twins that are alike, themselves
        z = torch.cat([z, z])
    z, u = z.to(dtype).to(DEV), torch.rand(3, generator=g).to(DEV)
    for kw in (dict(top_k=1), dict(top_k=2000), dict(top_k=2049), dict(top_k=11000), dict(top_p=0.3), dict(top_p=0.7, top_k=30000),
               dict(top_k=2048, top_p=0.5), dict(temperature=0.0), dict(min_p=0.2, top_p=0.99)):
        check(z, u, cfg_scale=cfg, **kw)


def test_long_rows_with_masks_and_infinities():
    z, u = rows_of(7, LONG, seed=33)
    z[0] = -INF
    z[1, 1:] = -INF
    z[2, 5:] = float("nan")
    z[3, 100:39000] = torch.finfo(torch.float32).min
    z[4, ::2] = -INF
    z[5, [7, 20001, LONG - 1]] = INF
    z[6, 3:] = -3.0e38
    for kw in (dict(), dict(top_k=20), dict(top_k=3000), dict(top_p=0.6), dict(min_p=0.2), dict(top_k=300, top_p=0.9, min_p=0.01), dict(temperature=0.0)):
        tokens = check(z, u, **kw)
        assert tokens[0] == -1 and tokens[1] == 0 and tokens[5] in (7, 20001, LONG - 1)


@pytest.mark.parametrize("cfg", [0.0, 4.0])
def test_long_rows_in_place(cfg):
    """The filtered logits in the place of the logits, which every pass reads again."""
    z, u = rows_of(4, LONG, seed=34)
    u = u[:2].contiguous() if cfg else u
    for kw in (dict(top_k=300, top_p=0.9), dict(top_k=2048), dict(temperature=0.7, top_k=5000), dict(temperature=0.8, top_p=0.9, min_p=1e-3), dict()):
        want = run(z, u, cfg_scale=cfg, **kw)
        again = z.clone()
        got = run(again, u, in_place=True, cfg_scale=cfg, **kw)
        assert all(np.array_equal(a, b) for a, b in zip(want, got))
        assert torch.equal(again[len(u):], z[len(u):])                     # the twins stay as they were


@pytest.mark.parametrize("V", [70000, 131072, 262144])
def test_large_vocabularies(V):
    z, u = rows_of(2, V, seed=V, spread=3.0)
    check(z, u, top_k=500, top_p=0.9)
    check(z, u, top_p=0.9, min_p=1e-3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cfg", [0.0, 4.0])
def test_filters_and_types(dtype, cfg):
    z, u = rows_of(8, 1500, seed=5, dtype=dtype)
    u = u[:4].contiguous() if cfg else u
    for T, k, p, m in itertools.product((0.0, 0.3, 1.0), (0, 1, 40, 1499, 1500, 5000), (1.0, 0.5, 1e-9), (0.0, 0.05, 1.0)):
        check(z, u, temperature=T, top_k=k, top_p=p, min_p=m, cfg_scale=cfg)


@pytest.mark.parametrize("scale", [0.3, 1.0, 2.7, 7.5])
def test_guidance_rounds_every_operation(scale):
    z, u = rows_of(8, 5000, seed=21)
    check(z, u[:4].contiguous(), cfg_scale=scale)
    check(z, u[:4].contiguous(), cfg_scale=scale, top_k=700, top_p=0.9)


def test_ties_go_to_the_lowest_index():
    g = torch.Generator().manual_seed(1)
    z = torch.randint(0, 4, (6, 3000), generator=g).float().to(DEV)          # about 750 entries of each value
    z[0] = 0.0                                                               # all alike
    z[1, 100:] = -0.0
    z[1, :100] = 0.0                                                         # the two zeros are one value
    u = torch.rand(6, generator=g).to(DEV)
    for k, p in ((1, 1.0), (10, 1.0), (800, 1.0), (0, 0.1), (0, 0.7), (900, 0.95), (900, 0.999), (751, 0.5), (2999, 0.9999)):
        check(z, u, top_k=k, top_p=p)
    tokens, _, out = run(z, u, temperature=0.0)
    assert tokens[0] == 0 and all((out[r] > -INF).sum() == 1 for r in range(6))


def test_masked_entries():
    z, u = rows_of(8, 700, seed=2)
    z[0] = -INF                                   # nothing to draw
    z[1, 1:] = -INF                               # one entry
    z[2, 5:] = float("nan")                       # NaN is masked
    z[3] = float("nan")
    z[4, 100:600] = torch.finfo(torch.float32).min
    z[5] = torch.finfo(torch.float32).min         # a mask of the type's lowest value over the whole row: a flat distribution
    z[6, ::2] = -INF
    z[7, 3:] = -3.0e38
    for kw in (dict(), dict(top_k=20), dict(top_p=0.6), dict(min_p=0.2), dict(top_k=300, top_p=0.9, min_p=0.01), dict(temperature=0.0), dict(temperature=1e-3)):
        tokens = check(z, u, **kw)
        assert tokens[0] == -1 and tokens[3] == -1 and tokens[1] == 0


def test_infinite_entries_share_the_mass():
    z, u = rows_of(2, 300, seed=3)
    z[0, [7, 200]] = INF
    u[0] = 0.75
    z[1, 9] = INF
    tokens, probs, out = run(z, u)
    assert np.isfinite(out).all()
    assert tokens[0] == 200 and tokens[1] == 9
    assert probs[0, 7] == 0.5 and probs[0, 200] == 0.5 and probs[1, 9] == 1.0 and probs.sum() == 2.0


def test_uniforms_at_and_beyond_the_ends():
    z, _ = rows_of(1, 100, seed=4)
    z = z.repeat(6, 1)
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, -1.0, float("nan"), INF], device=DEV)
    tokens = check(z, u)
    assert tokens[0] == 0 and tokens[3] == 0 and tokens[4] == 0 and tokens[1] == tokens[2] == tokens[5]


def test_strides_alignment_and_outputs_in_place():
    z, u = rows_of(5, 1001, seed=6)
    kw = dict(temperature=0.8, top_k=300, top_p=0.9)
    want = run(z, u, **kw)
    wide = torch.full((5, 1301), 50.0, device=DEV)
    for first in (0, 1, 3):
        wide.fill_(50.0)
        wide[:, first:first + 1001] = z
        got = run(wide[:, first:first + 1001], u, **kw)
        assert all(np.array_equal(a, b) for a, b in zip(want, got))
    got = run(z.clone(), u, in_place=True, **kw)
    assert all(np.array_equal(a, b) for a, b in zip(want, got))
    zz, uu = rows_of(6, 1000, seed=7)
    want = run(zz, uu[:3].contiguous(), cfg_scale=4.0, **kw)
    got = run(zz, uu[:3].contiguous(), in_place=True, cfg_scale=4.0, **kw)
    assert all(np.array_equal(a, b) for a, b in zip(want, got))
    # bf16 rows that begin anywhere
    zb, ub = rows_of(4, 1501, seed=8, dtype=torch.bfloat16)
    check(zb, ub, **kw)
    wb = torch.full((4, 1603), 50.0, dtype=torch.bfloat16, device=DEV)
    for first in (1, 2, 3):
        wb[:, first:first + 1501] = zb
        got = run(wb[:, first:first + 1501], ub, **kw)
        assert all(np.array_equal(a, b) for a, b in zip(run(zb, ub, **kw), got))
    # outputs one at a time
    p = mulo.make_sample_params(**kw)
    want = run(z, u, **kw)
    t, pr, lo = torch.empty(5, dtype=torch.int32, device=DEV), torch.empty(5, 1001, device=DEV), torch.empty(5, 1001, device=DEV)
    mulo.mulo_sample_filtered(p, z, u, tokens=t)
    mulo.mulo_sample_filtered(p, z, probs=pr)
    mulo.mulo_sample_filtered(p, z, logits_out=lo)
    torch.cuda.synchronize()
    assert np.array_equal(t.cpu().numpy(), want[0]) and np.array_equal(pr.cpu().numpy(), want[1]) and np.array_equal(lo.cpu().numpy(), want[2])


def test_skewed_values():
    """Values far apart, a few large outliers over a dense bulk, and a bulk that float32 hardly tells apart: the search for the
    border may not rely on how values are spread."""
    g = torch.Generator().manual_seed(8)
    V = 5000
    z = torch.empty(6, V)
    z[0] = torch.randn(V, generator=g) * 1e4
    z[1] = torch.randn(V, generator=g) * 1e-5
    z[1, 17] = 1000.0
    z[2] = 1.0 + torch.randint(0, 3, (V,), generator=g) * 2.0 ** -23
    z[3] = torch.randn(V, generator=g) * 1e30
    z[4] = torch.randn(V, generator=g) * 1e-38
    z[5] = -torch.rand(V, generator=g).pow(8) * 100
    z, u = z.to(DEV), torch.rand(6, generator=g).to(DEV)
    for kw in (dict(), dict(top_k=1), dict(top_k=37), dict(top_k=2500), dict(top_p=0.3), dict(top_p=0.999), dict(top_k=1000, top_p=0.9), dict(min_p=0.1)):
        check(z, u, **kw)


@pytest.mark.parametrize("top", [0.75, 1.5, 10.0, 100.0, 10000.0, -10.0])
@pytest.mark.parametrize("T", [1e-6, 1e-8, 1e-9, 1e-10, 1e-20, 1e-30])
def test_small_temperatures(top, T):
    """Steps of float32 that are hundreds of bits and more: the entry a step below the largest weighs nothing, whichever way
    a limit between the two would be rounded."""
    z = torch.full((1, 300), top)
    for i in range(1, 300):
        z[0, i] = torch.nextafter(z[0, i - 1], torch.tensor(-INF)) if i % 3 else z[0, i - 1]
    order = torch.randperm(300, generator=torch.Generator().manual_seed(12))
    z = torch.cat([z, z[:, order], z.flip(1)]).to(DEV)
    u = torch.tensor([0.0, 0.6, 0.9], device=DEV)
    for kw in (dict(), dict(top_k=5), dict(top_k=250), dict(top_p=0.9), dict(min_p=1e-3), dict(top_k=7, top_p=0.5)):
        check(z, u, temperature=T, **kw)


def test_distribution_of_draws():
    """Uniforms on a grid land on every entry in proportion to its probability."""
    z, _ = rows_of(1, 50, seed=9)
    n = 4096
    u = (torch.arange(n, dtype=torch.float32) / n).to(DEV)
    p = mulo.make_sample_params(top_k=30, top_p=0.95)
    tokens, probs = torch.empty(n, dtype=torch.int32, device=DEV), torch.empty(n, 50, device=DEV)
    mulo.mulo_sample_filtered(p, z.repeat(n, 1), u, tokens, probs)
    counts = torch.bincount(tokens.long(), minlength=50).double() / n
    assert (counts - probs[0].double()).abs().max().item() <= 1.0 / n + 1e-6      # a grid of n points: off by at most one each


def test_captured_and_replayed():
    z, u = rows_of(4, 3000, seed=10)
    p = mulo.make_sample_params(temperature=0.9, top_k=500, top_p=0.9)
    side = torch.cuda.Stream()
    tokens = torch.empty(4, dtype=torch.int32, device=DEV)
    with torch.cuda.stream(side):
        mulo.mulo_sample_filtered(p, z, u, tokens)
        side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        mulo.mulo_sample_filtered(p, z, u, tokens)
    with torch.cuda.stream(side):
        for seed in (11, 12, 13):
            z2, u2 = rows_of(4, 3000, seed=seed)
            z.copy_(z2)
            u.copy_(u2)
            tokens.fill_(-7)
            graph.replay()
            side.synchronize()
            assert np.array_equal(tokens.cpu().numpy(), run(z2, u2, temperature=0.9, top_k=500, top_p=0.9)[0])
    del graph
    say("  3 replays")
