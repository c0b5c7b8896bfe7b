"""A context with an attached prefix, with a window, and the operators as a serving program runs them together."""
import numpy as np
import pytest
import torch

import paper_2601_05149_amd as mulo
from oracle import decoder as OD
from oracle import sampling as OS
from oracle import step as ST
from tests.gpu_util import DEV, check_bf16_logits, compare_decisions, decide_buffers, make_ctx, say, to_np
from workloads import generators as G

pytestmark = pytest.mark.gpu
TINY = dict(n_layers=2, d_model=256, n_heads=4, head_dim=64, d_ffn=688, vocab=1024, dtype="f32", rms_eps=1e-5)
SMALL = dict(n_layers=2, d_model=512, n_heads=8, head_dim=64, d_ffn=1408, vocab=2048, dtype="bf16", rms_eps=1e-5)
WIDE = dict(n_layers=1, d_model=512, n_heads=4, head_dim=128, d_ffn=1408, vocab=2048, dtype="bf16", rms_eps=1e-5)
MODELS = dict(tiny=TINY, small=SMALL, wide=WIDE)


def dev(a):
    return torch.tensor(np.ascontiguousarray(a), device=DEV)


def forward(ctx, kv, tokens, P):
    B, L = tokens.shape
    z = torch.full((B, L, ctx.cfg.vocab), float("nan"), device=DEV)
    mulo.mulo_verify_forward(ctx, kv, B, L, P, dev(tokens), None, z)
    torch.cuda.synchronize()
    return z.cpu().numpy()


def with_prefix(m, w, prefix, B, max_seq, max_block, groups=None, copy=False):
    """A context of B sequences over the prefixes `prefix` [G, S], which another context of the same weights fills."""
    G_, S = prefix.shape
    cp, _, _ = make_ctx(m, w, G_, (S + 7) // 8 * 8, (S + 3) // 4 * 4)
    kvp = mulo.alloc_kv(cp, DEV)
    forward(cp, kvp, prefix, 0)
    ctx, _, _ = make_ctx(m, w, B, max_seq, max_block, stream_copy=copy)
    cos, sin = G.rope_table(S + max_seq, m["head_dim"])
    kv = mulo.alloc_kv(ctx, DEV)
    mulo.mulo_attach_prefix(ctx, kvp, S, dev(cos[S:]), dev(sin[S:]))
    return ctx, kv, cos, sin, cp


def oracle(m, w, cos, sin, B, rows, round_bf16, sinks=0, window=0):
    d = OD.DecoderOracle(m, w, cos, sin, B, rows, round_bf16=round_bf16)
    d.sinks, d.window = sinks, window
    return d


@pytest.mark.parametrize("name, B, groups, S, sinks, window, copy", [
    ("tiny", 3, 1, 33, 0, 0, False), ("tiny", 4, 2, 50, 10, 37, False), ("small", 4, 2, 77, 0, 0, False), ("small", 3, 1, 40, 5, 30, False),
    ("wide", 6, 1, 64, 0, 0, True), ("wide", 2, 2, 65, 70, 20, False),
    ("wide", 16, 2, 1300, 0, 0, False), ("wide", 16, 1, 1300, 900, 1200, False)])      # long enough for the sequences to be stacked over it
def test_forward_behind_a_shared_prefix(name, B, groups, S, sinks, window, copy):
    """Blocks and single tokens behind a shared prefix: what a decoder computes whose every sequence begins with the prefix."""
    m = MODELS[name]
    w = G.make_weights(m, seed=0)
    L = [140, 12, 1, 1]
    rows = (sum(L) + 7) // 8 * 8
    prefix = G.uniform_tokens((groups, S), m["vocab"], 0, tag=0)
    ctx, kv, cos, sin, _ = with_prefix(m, w, prefix, B, rows, 160, copy=copy)
    mulo.mulo_set_window(ctx, sinks, window)
    bf16 = m["dtype"] == "bf16"
    # the prefix itself was filled without a window: so is the oracle's
    decs = [oracle(m, w, cos, sin, B, S + rows, r) for r in ((True, False) if bf16 else (False,))]
    whole = np.repeat(prefix, B // groups, 0)
    for d in decs:
        d.forward(whole, 0)
        d.sinks, d.window = sinks, window
    P = 0
    for i, n in enumerate(L):
        toks = G.uniform_tokens((B, n), m["vocab"], 1, tag=i)
        z = forward(ctx, kv, toks, P)
        want = [d.forward(toks, S + P).numpy() for d in decs]
        if bf16:
            check_bf16_logits("%s, %d tokens at %d" % (name, n, P), z, *want)
        else:
            err = np.abs(z - want[0]).max()
            say("  %s, %d tokens at %d: %.3g" % (name, n, P, err))
            assert err <= 1e-4
        P += n


@pytest.mark.parametrize("name", ["tiny", "small"])
def test_forward_through_a_window(name):
    m = MODELS[name]
    w = G.make_weights(m, seed=0)
    B, L, rows = 2, [70, 150, 3, 1], 232
    ctx, cos, sin = make_ctx(m, w, B, rows, 152)
    kv = mulo.alloc_kv(ctx, DEV)
    mulo.mulo_set_window(ctx, 6, 40)
    bf16 = m["dtype"] == "bf16"
    decs = [oracle(m, w, cos, sin, B, rows, r, 6, 40) for r in ((True, False) if bf16 else (False,))]
    P = 0
    for i, n in enumerate(L):
        toks = G.uniform_tokens((B, n), m["vocab"], 1, tag=i)
        z = forward(ctx, kv, toks, P)
        want = [d.forward(toks, P).numpy() for d in decs]
        if bf16:
            check_bf16_logits("%s, %d tokens at %d" % (name, n, P), z, *want)
        else:
            assert np.abs(z - want[0]).max() <= 1e-4
        P += n


def test_detached_and_without_a_window_nothing_is_left():
    m = SMALL
    w = G.make_weights(m, seed=0)
    prefix, toks = G.uniform_tokens((1, 24), m["vocab"], 0, tag=0), G.uniform_tokens((2, 40), m["vocab"], 1, tag=0)
    ctx, kv, cos, sin, _ = with_prefix(m, w, prefix, 2, 64, 48)
    mulo.mulo_set_window(ctx, 1, 5)
    seen = forward(ctx, kv, toks, 0)
    mulo.mulo_attach_prefix(ctx)
    mulo.mulo_set_window(ctx, 0, 0)
    back = forward(ctx, kv, toks, 0)
    plain, _, _ = make_ctx(m, w, 2, 64, 48)
    assert np.array_equal(back, forward(plain, mulo.alloc_kv(plain, DEV), toks, 0)) and not np.array_equal(back, seen)


@pytest.mark.parametrize("B, S", [(3, 41), (24, 1300)])
def test_resampling_behind_a_prefix(B, S):
    """One pass over scattered islands, and single tokens in order, behind an attached prefix: the logits of a context whose
    sequences hold the prefix themselves (one layer: the same inputs up to the attention, whose sums are the same terms)."""
    m = WIDE
    w = G.make_weights(m, seed=0)
    H, W = 4, 8
    L = H * W
    prefix = G.uniform_tokens((1, S), m["vocab"], 0, tag=0)
    toks, prev = G.uniform_tokens((B, L), m["vocab"], 1, tag=0), G.uniform_tokens((B,), m["vocab"], 2, tag=0)
    mask = np.zeros((B, L), np.uint8)
    mask[0, [3, 17, 30]] = 1
    mask[1, [9]] = 1
    mask[2, [0, 21]] = 1
    mask[3:, [2, 28]] = 1
    ctx, kv, cos, sin, _ = with_prefix(m, w, prefix, B, L, L)
    rows = (S + L + 7) // 8 * 8
    full, _, _ = make_ctx(m, w, B, rows, (S + 3) // 4 * 4 + 4)
    kvf = mulo.alloc_kv(full, DEV)
    forward(full, kvf, np.repeat(prefix, B, 0), 0)
    for window in (0, 20):
        for c in (ctx, full):
            mulo.mulo_set_window(c, 4, window)
        got = []
        for c, cache, P in ((ctx, kv, 0), (full, kvf, S)):
            forward(c, cache, np.concatenate([prev[:, None], toks[:, :-1]], 1), P)
            i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device=DEV)
            island, rank, counts = i32(B, L), i32(B, L), i32(B, 2)
            mulo.mulo_rejection_islands(c, B, W, 0, L, dev(mask), island, rank, counts)
            t, z, over = dev(toks), torch.zeros(B, L, m["vocab"], device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
            mulo.mulo_resample_islands(c, cache, B, P, L, 1, 3, 5, 7, dev(prev), dev(mask), rank, t, z, over)
            zs = torch.zeros(B, L, m["vocab"], device=DEV)
            mulo.mulo_resample_sequential(c, cache, B, P, L, L - 2, 5, 7, dev(prev), dev(np.zeros((B, L), np.uint8)), dev(toks), zs)
            torch.cuda.synchronize()
            assert int(over) == 0
            got.append((z.cpu().numpy(), zs.cpu().numpy()))
        for a, b, what in zip(got[0], got[1], ("islands", "in order")):
            assert np.abs(b).max() > 0.1
            say("  window %d, %s: %.3g" % (window, what, np.abs(a - b).max()))
            assert np.abs(a - b).max() <= 2e-2


@pytest.mark.parametrize("name, B, S, sinks, window, cfg_scale", [
    ("tiny", 2, 33, 0, 0, 0.0), ("tiny", 2, 50, 10, 37, 4.0), ("small", 3, 77, 0, 0, 0.0), ("small", 2, 40, 5, 30, 4.0),
    ("wide", 4, 65, 70, 20, 0.0), ("wide", 2, 300, 0, 0, 4.0)])
def test_verification_step_behind_a_prefix_and_through_a_window(name, B, S, sinks, window, cfg_scale):
    """A whole step, plain and guided (the prompt and the empty prompt as two prefixes), in front of 8 committed rows: the logits of a
    decoder whose every sequence begins with its prefix, the bits of its stages called one by one, and the decisions of the oracle on
    those logits."""
    m = MODELS[name]
    w = G.make_weights(m, seed=0)
    H, W, r, V, P = 16, 8, 2, m["vocab"], 8
    L, n_lo = H * W, H * W // 4
    Bz, groups = (2 * B, 2) if cfg_scale else (B, 1)
    prefix = G.uniform_tokens((groups, S), V, 0, tag=0)
    ctx, kv, cos, sin, _ = with_prefix(m, w, prefix, Bz, P + L, L)
    mulo.mulo_set_window(ctx, sinks, window)
    before = np.concatenate([G.uniform_tokens((B, P), V, 0, tag=1)] * (Bz // B))
    forward(ctx, kv, before, 0)
    dl = G.normal_logits((B, n_lo, V), 1.0, 0, tag=2)
    dt, prev = dev(G.sample_categorical(dl, 0, tag=2)), dev(before[:B, -1])
    dl = dev(dl)
    p = mulo.make_params(H, W, 0, L, 1, seed=3, rng_counter=4, cfg_scale=cfg_scale)
    i32 = lambda *shape: torch.empty(*shape, dtype=torch.int32, device=DEV)
    out, toks, z = decide_buffers(B, L), i32(B, L), torch.empty(Bz, L, V, device=DEV)
    mulo.mulo_verify_step(ctx, kv, B, P, p, H // r, W // r, r, dl, 0, dt, prev, out["tokens_out"], out["accept"], out["mask"], out["t0"],
                          out["stats"], toks, z)
    toks2, q, q_row, z2, out2 = i32(B, L), torch.empty(B, n_lo, V, device=DEV), i32(L), torch.empty(Bz, L, V, device=DEV), decide_buffers(B, L)
    mulo.mulo_upsample_draft(ctx, B, H // r, W // r, r, dl, 0, dt, toks2, q, q_row, None)
    rows = torch.cat([torch.cat([prev[:, None], toks2[:, :-1]], 1)] * (Bz // B))
    mulo.mulo_verify_forward(ctx, kv, Bz, L, P, rows, None, z2)
    mulo.mulo_accept_local_resample(ctx, B, p, z2, q, q_row, n_lo * V, toks2, **out2)
    torch.cuda.synchronize()
    assert torch.equal(z, z2) and torch.equal(toks, toks2)
    for k in out:
        assert torch.equal(out[k], out2[k]), k
    bf16 = m["dtype"] == "bf16"
    want = []
    for rounded in ((True, False) if bf16 else (False,)):
        d = oracle(m, w, cos, sin, Bz, S + P + L, rounded)
        d.forward(np.repeat(prefix, Bz // groups, 0), 0)
        d.sinks, d.window = sinks, window
        d.forward(before, S)
        want.append(d.forward(rows.cpu().numpy(), S + P).numpy())
    zh = z.cpu().numpy()
    if bf16:
        check_bf16_logits("step, %s" % name, zh, *want)
    else:
        say("  step, %s: %.3g" % (name, np.abs(zh - want[0]).max()))
        assert np.abs(zh - want[0]).max() <= 1e-4
    guided = dict(logits_uncond=zh[B:], cfg_scale=cfg_scale) if cfg_scale else {}
    ref = ST.decide(zh[:B], q.cpu().numpy(), q_row.cpu().numpy(), toks.cpu().numpy(), W=W, n0=0, radius=1, seed=3, rng_counter=4, **guided)
    say("  %r" % compare_decisions(to_np(out), ref, toks.cpu().numpy(), q.cpu().numpy(), q_row.cpu().numpy(), label="step"))
    assert 0 < ref["accept"].sum() < B * L


def test_a_step_behind_a_prefix_recorded_and_replayed():
    """One graph of a step behind a shared prefix and through a window, replayed over other drafts: the bits of an ordinary call."""
    m = SMALL
    w = G.make_weights(m, seed=0)
    B, S, H, W, r, V, P = 8, 600, 8, 8, 2, m["vocab"], 8
    L, n_lo = H * W, H * W // 4
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx, kv, _, _, cp = with_prefix(m, w, G.uniform_tokens((1, S), V, 0, tag=0), B, P + L, L)
        mulo.mulo_set_window(ctx, 5, 400)
        before = G.uniform_tokens((B, P), V, 0, tag=1)
        forward(ctx, kv, before, 0)
        prev, dl, dt = dev(before[:, -1]), torch.zeros(B, n_lo, V, device=DEV), torch.zeros(B, n_lo, dtype=torch.int32, device=DEV)
        out, z = decide_buffers(B, L), torch.empty(B, L, V, device=DEV)
        p = mulo.make_params(H, W, 0, L, 1, seed=3, rng_counter=4)

        def step():
            mulo.mulo_verify_step(ctx, kv, B, P, p, H // r, W // r, r, dl, 0, dt, prev, logits=z, **out)

        step()
        side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    with torch.cuda.stream(side):
        for tag in (2, 3, 4):
            drawn = G.normal_logits((B, n_lo, V), 1.0, 0, tag=tag)
            dl.copy_(torch.tensor(drawn))
            dt.copy_(torch.tensor(G.sample_categorical(drawn, 0, tag=tag)))
            got = []
            for run in (graph.replay, step):
                for t in list(out.values()) + [z]:
                    t.fill_(77)
                run()
                side.synchronize()
                got.append([t.clone() for t in list(out.values()) + [z]])
            assert all(torch.equal(a, b) for a, b in zip(*got))
            assert 0 < int(out["accept"].sum()) < B * L
    del graph


def test_groups_have_to_divide_the_batch():
    m = WIDE
    w = G.make_weights(m, seed=0)
    ctx, kv, *_ = with_prefix(m, w, G.uniform_tokens((2, 16), m["vocab"], 0, tag=0), 4, 16, 16)
    z = torch.empty(4, 8, m["vocab"], device=DEV)
    with pytest.raises(mulo.MuloError) as e:
        mulo.mulo_verify_forward(ctx, kv, 3, 8, 0, dev(np.zeros((3, 8), np.int32)), None, z)
    assert e.value.status == 2
    with pytest.raises(mulo.MuloError) as e:
        mulo.mulo_set_window(ctx, 0, -1)
    assert e.value.status == 3


def test_a_guided_block_as_it_is_served():
    """Two images of one prompt with guidance: the prompt and the empty prompt are two shared prefixes, the model looks through
    a window, the draft is drawn from a filtered distribution, the target's guided logits are filtered the same way
    and go through the accept test; then one token more.  Every stage against its oracle on the stage's own inputs."""
    m = SMALL
    w = G.make_weights(m, seed=0)
    B, S, H, W, V = 2, 30, 8, 8, m["vocab"]
    L = H * W
    prefix = G.uniform_tokens((2, S), V, 0, tag=0)
    ctx, kv, cos, sin, _ = with_prefix(m, w, prefix, 2 * B, L + 8, L)
    mulo.mulo_set_window(ctx, 20, 48)
    u = torch.rand(B * L, generator=torch.Generator().manual_seed(1)).to(DEV)
    # the drafter's rows: a token and its distribution
    dl = dev(G.normal_logits((B * L, V), 2.0, 0, tag=3))
    filt = dict(temperature=0.9, top_k=200, top_p=0.95, min_p=0.002)
    draft, q = torch.empty(B * L, dtype=torch.int32, device=DEV), torch.empty(B * L, V, device=DEV)
    mulo.mulo_sample_filtered(mulo.make_sample_params(**filt), dl, u, draft, q)
    prev = G.uniform_tokens((B,), V, 2, tag=0)
    toks = draft.cpu().numpy().reshape(B, L)
    rows = np.concatenate([prev[:, None], toks[:, :-1]], 1)
    z = torch.empty(2 * B, L, V, device=DEV)
    mulo.mulo_verify_forward(ctx, kv, 2 * B, L, 0, dev(np.concatenate([rows, rows])), None, z)
    decs = []
    for r in (True, False):
        d = oracle(m, w, cos, sin, 2 * B, S + L + 8, r)
        d.forward(np.repeat(prefix, B, 0), 0)
        d.sinks, d.window = 20, 48
        decs.append(d.forward(np.concatenate([rows, rows]), S).numpy())
    torch.cuda.synchronize()
    check_bf16_logits("guided block", z.cpu().numpy(), *decs)
    zk = torch.empty(B * L, V, device=DEV)
    tf = dict(temperature=0.8, top_k=500, top_p=0.98)
    mulo.mulo_sample_filtered(mulo.make_sample_params(cfg_scale=4.0, **tf), z.reshape(2 * B * L, V), logits_out=zk)
    out = decide_buffers(B, L)
    p = mulo.make_params(H, W, 0, L, 1, resample_mode=0, seed=3, rng_counter=4)
    mulo.mulo_accept_local_resample(ctx, B, p, zk.reshape(B, L, V), q.reshape(B, L, V), None, L * V, draft.reshape(B, L), **out)
    torch.cuda.synchronize()
    kept = zk.cpu().numpy()
    guided = OS.row_logits(z.reshape(2 * B * L, V).cpu().numpy(), 4.0)
    for r in range(0, B * L, 7):
        assert np.array_equal(np.nonzero(np.isfinite(kept[r]))[0], sorted(OS.kept(guided[r], **tf)))
        assert np.array_equal(np.nonzero(q[r].cpu().numpy())[0], sorted(OS.kept(dl[r].cpu().numpy(), **filt)))
    ref = ST.decide(kept.reshape(B, L, V).astype(np.float64), q.cpu().numpy().reshape(B, L, V), None, toks, W=W, n0=0, radius=1, seed=3, rng_counter=4)
    acc = out["accept"].cpu().numpy()
    assert not ((acc != ref["accept"]) & ~ref["near_tie"]).any() and 0 < acc.sum() < B * L
    got, mask = out["tokens_out"].cpu().numpy(), out["mask"].cpu().numpy().astype(bool)
    assert mask.any() and np.isfinite(kept[np.arange(B * L), got.reshape(-1)].reshape(B, L)[mask]).all()      # re-draws lie in what stays
    if np.array_equal(acc, ref["accept"]):
        assert np.array_equal(mask, ref["mask"].astype(bool)) and (got == ref["tokens_out"]).mean() > 0.99
    # commit, and draw the token behind the block
    rows = np.concatenate([prev[:, None], got[:, :-1]], 1)
    mulo.mulo_verify_forward(ctx, kv, 2 * B, L, 0, dev(np.concatenate([rows, rows])), None, z)
    last = dev(np.concatenate([got[:, -1:], got[:, -1:]]))
    z1, t1 = torch.empty(2 * B, 1, V, device=DEV), torch.empty(B, dtype=torch.int32, device=DEV)
    mulo.mulo_verify_forward(ctx, kv, 2 * B, 1, L, last, None, z1)
    mulo.mulo_sample_filtered(mulo.make_sample_params(cfg_scale=4.0, **tf), z1.reshape(2 * B, V), u[:B].contiguous(), t1)
    torch.cuda.synchronize()
    g1 = OS.row_logits(z1.reshape(2 * B, V).cpu().numpy(), 4.0)
    for b in range(B):
        tok, far = OS.draw(OS.kept(g1[b], **tf), float(u[b]))
        assert int(t1[b]) == tok or far < V * 2.0 ** -45
