"""CPU-side checks of mulo_attention, mulo_attach_prefix, mulo_set_window and mulo_sample_filtered: what they refuse, before
anything touches a GPU, and their oracle's own pins."""
import ctypes as C
import math
import os

import numpy as np
import pytest
import torch

import paper_2601_05149_amd as mulo
from oracle import context as OC
from oracle import sampling as OS
from paper_2601_05149_amd import binding as BD

NULL, SHAPE, RANGE, UNSUPPORTED = 1, 2, 3, 6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(BD.LIB_PATH):
        from paper_2601_05149_amd import build
        build.build_lib()
    return mulo.load_library()


def attention_args(**changes):
    """Arguments that hold (pointers that nothing follows), with changes."""
    a = BD.AttentionArgs(dtype=1, B=4, L=2, n_heads=8, n_kv_heads=2, head_dim=64, q=256, q_batch=1024, q_head=128, q_row=64, out=512,
                         out_batch=1024, out_head=64, out_row=512, k=1024, v=2048, k_batch=8192, k_head=4096, k_row=64, v_batch=8192,
                         v_head=4096, v_chan=64, rows=64, P=62, prefix_k=4096, prefix_v=8192, prefix_k_group=8192, prefix_k_head=4096,
                         prefix_k_row=64, prefix_v_group=8192, prefix_v_head=4096, prefix_v_chan=64, n_prefix=2, prefix_len=61,
                         prefix_rows=64, sinks=3, window=9, scale=0.0)
    for name, value in changes.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("status, changes", [
    (0, {}), (0, dict(window=0)), (0, dict(sinks=2 ** 31 - 1, window=2 ** 31 - 1)), (0, dict(k_batch=0, v_batch=0)),
    (0, dict(prefix_len=0, prefix_k=None, prefix_v=None, n_prefix=0, prefix_rows=0, prefix_k_group=-3)),
    (NULL, dict(q=None)), (NULL, dict(out=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(prefix_k=None)), (NULL, dict(prefix_v=None)),
    (RANGE, dict(dtype=2)), (RANGE, dict(B=0)), (RANGE, dict(L=0)), (RANGE, dict(n_heads=0)), (RANGE, dict(n_kv_heads=0)), (RANGE, dict(P=-1)),
    (RANGE, dict(rows=0)), (RANGE, dict(prefix_len=-1)), (RANGE, dict(sinks=-1)), (RANGE, dict(window=-1)), (RANGE, dict(n_prefix=0)),
    (RANGE, dict(scale=-1.0)), (RANGE, dict(scale=math.nan)), (RANGE, dict(scale=math.inf)), (RANGE, dict(scale=1.1e6)), (RANGE, dict(q_batch=-8)), (RANGE, dict(v_chan=1 << 41)),
    (SHAPE, dict(P=63)), (SHAPE, dict(n_kv_heads=3)), (SHAPE, dict(n_prefix=3)), (SHAPE, dict(prefix_len=65)), (SHAPE, dict(k_row=32)),
    (SHAPE, dict(v_chan=56)), (SHAPE, dict(prefix_k_row=56)), (SHAPE, dict(prefix_v_chan=56)),
    # outputs on top of each other
    (SHAPE, dict(out_batch=0)), (SHAPE, dict(out_head=32)), (SHAPE, dict(out_row=64)), (SHAPE, dict(out_batch=512)),
    (0, dict(out_batch=64, out_head=512, out_row=256, B=4, L=2)), (0, dict(L=1, out_row=0)),
    (UNSUPPORTED, dict(head_dim=32, q_row=64)), (UNSUPPORTED, dict(q_row=68)), (UNSUPPORTED, dict(k_batch=8193)), (UNSUPPORTED, dict(rows=62, P=0)),
    (UNSUPPORTED, dict(prefix_rows=63)), (UNSUPPORTED, dict(q=264)), (UNSUPPORTED, dict(out=8)), (UNSUPPORTED, dict(v=2052)),
    (UNSUPPORTED, dict(prefix_k=4100)), (UNSUPPORTED, dict(k_row=1 << 23)), (UNSUPPORTED, dict(B=1 << 28, n_prefix=1, out_batch=1024)),
    (UNSUPPORTED, dict(B=1 << 20, n_prefix=1)), (0, dict(B=1 << 19, n_prefix=1)),
    (UNSUPPORTED, dict(B=1 << 19, L=16, P=0, n_prefix=1, out_batch=8192)), (0, dict(B=1 << 18, L=16, P=0, n_prefix=1, out_batch=8192)),
    (0, dict(dtype=0)), (0, dict(dtype=0, q_row=68)), (UNSUPPORTED, dict(dtype=0, q_row=66)), (0, dict(dtype=0, rows=60, P=0)),
], ids=str)
def test_attention_arguments(lib, status, changes):
    a = attention_args(**changes)
    assert lib.mulo_check_attention(C.byref(a)) == status
    if status:
        assert lib.mulo_attention(None, C.byref(a), None, 0) == status
        assert lib.mulo_attention_workspace_bytes(C.byref(a)) == 0


def test_attention_without_arguments(lib):
    assert lib.mulo_check_attention(None) == NULL and lib.mulo_attention(None, None, None, 0) == NULL
    assert lib.mulo_attention(None, C.byref(attention_args()), C.c_void_p(8), 64) == UNSUPPORTED       # a workspace off its 16 bytes


def test_the_workspace_is_bounded(lib):
    """Partial results take less than the caches they come from would, or little."""
    for B, L, P, S in ((1, 1, 8000, 0), (64, 1, 900, 2048), (16, 16, 330, 4224), (4, 1024, 2048, 1024), (1, 64, 30000, 0)):
        a = attention_args(B=B, L=L, n_heads=32, n_kv_heads=32, head_dim=128, rows=(P + L + 7) // 8 * 8, P=P, prefix_len=S, prefix_rows=S, n_prefix=1, window=0)
        for s in ("q_batch", "q_head", "q_row", "out_batch", "out_head", "out_row", "k_batch", "k_head", "k_row", "v_batch", "v_head", "v_chan"):
            setattr(a, s, 0)
        a.q_row = a.k_row = a.prefix_k_row = 128
        a.v_chan, a.prefix_v_chan = a.rows, max(a.prefix_rows, 8)
        a.out_head, a.out_row, a.out_batch = 128, 4096, 4096 * L
        assert lib.mulo_check_attention(C.byref(a)) == 0
        assert lib.mulo_attention_workspace_bytes(C.byref(a)) <= 64 << 20


def test_prefix_and_window_need_a_context(lib):
    assert lib.mulo_attach_prefix(None, None) == NULL and lib.mulo_set_window(None, 0, 0) == NULL


@pytest.mark.parametrize("status, changes, call", [
    (NULL, {}, dict(logits=None)), (NULL, {}, dict(u=None)), (NULL, {}, dict(tokens=None)),
    (RANGE, {}, dict(rows=0)), (RANGE, {}, dict(vocab=0)), (RANGE, {}, dict(dtype=2)),
    (RANGE, dict(temperature=-1.0), {}), (RANGE, dict(temperature=math.nan), {}), (RANGE, dict(temperature=math.inf), {}),
    (RANGE, dict(temperature=1e-31), {}), (RANGE, dict(top_k=-1), {}), (RANGE, dict(top_p=0.0), {}), (RANGE, dict(top_p=1.1), {}),
    (RANGE, dict(top_p=math.nan), {}), (RANGE, dict(min_p=-0.1), {}), (RANGE, dict(min_p=1.5), {}), (RANGE, dict(cfg_scale=-1.0), {}),
    (RANGE, dict(cfg_scale=math.nan), {}), (UNSUPPORTED, {}, dict(vocab=262145, stride=262145)), (SHAPE, {}, dict(stride=99)),
    (UNSUPPORTED, {}, dict(rows=1 << 22)),
    (SHAPE, {}, dict(stride=1 << 41)), (UNSUPPORTED, {}, dict(logits=258)), (UNSUPPORTED, {}, dict(dtype=1, logits=257)),
    (UNSUPPORTED, {}, dict(probs=1025)), (SHAPE, {}, dict(kept=256, dtype=1)), (SHAPE, {}, dict(kept=256, stride=104)),
    (SHAPE, {}, dict(probs=256)), (SHAPE, {}, dict(probs=1024, kept=1024)),
], ids=str)
def test_sample_arguments(lib, status, changes, call):
    p = mulo.make_sample_params(**changes)
    c = dict(dict(rows=2, vocab=100, dtype=0, logits=256, stride=100, u=512, tokens=768, probs=None, kept=None), **call)
    assert lib.mulo_sample_filtered(None, C.byref(p), c["rows"], c["vocab"], c["dtype"], c["logits"], c["stride"], c["u"], c["tokens"],
                                    c["probs"], c["kept"]) == status
    assert lib.mulo_sample_filtered(None, None, 2, 100, 0, 256, 100, 512, 768, None, None) == NULL


def test_binding_refuses_what_does_not_fit():
    t = torch.zeros(1, 2, 1, 64)
    with pytest.raises(ValueError):
        mulo.make_attention(t, t, t, t, 0)
    with pytest.raises(ValueError):
        mulo.mulo_sample_filtered(mulo.make_sample_params(), torch.zeros(2, 3))          # not on a GPU
    with pytest.raises(ValueError):
        mulo.mulo_sample_filtered(mulo.make_sample_params(), torch.zeros(2, 3, dtype=torch.float16))


def test_a_prefix_without_its_rotary_tables_is_refused():
    ctx = mulo.Ctx(None, mulo.make_cfg(dict(n_layers=1, d_model=128, n_heads=2, head_dim=64, d_ffn=128, vocab=64, dtype="bf16"), 2, 16, 8), [])
    k, v, table = torch.zeros(1, 1, 2, 24, 64).bfloat16(), torch.zeros(1, 1, 2, 64, 24).bfloat16(), torch.zeros(16, 32)
    for tables in ((None, None), (table, None), (None, table)):
        with pytest.raises(ValueError):
            mulo.mulo_attach_prefix(ctx, (k, v), 20, *tables)
    with pytest.raises(ValueError):
        mulo.mulo_attach_prefix(ctx, (k, v), 20, table, table)            # not on a GPU


# ---- the oracle --------------------------------------------------------------------------------------------------------
def test_oracle_attention_is_causal_softmax_attention():
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(2, 4, 6, 8, generator=g, dtype=torch.float64) for _ in range(3))
    pk, pv = torch.randn(1, 4, 5, 8, generator=g, dtype=torch.float64), torch.randn(1, 4, 5, 8, generator=g, dtype=torch.float64)
    want = torch.nn.functional.scaled_dot_product_attention(
        q, torch.cat([pk.expand(2, -1, -1, -1), k], 2), torch.cat([pv.expand(2, -1, -1, -1), v], 2),
        attn_mask=torch.arange(11)[None, :] <= 5 + torch.arange(6)[:, None])
    out = OC.context_attention(q, k, v.transpose(2, 3), [0, 0], pk, pv.transpose(2, 3), 5)[0]
    assert (out - want).abs().max() < 1e-12
    # a window of everything changes nothing, a window of one is the value itself, sinks come back
    assert torch.equal(OC.context_attention(q, k, v.transpose(2, 3), [0, 0], pk, pv.transpose(2, 3), 5, 0, 11)[0], out)
    assert torch.allclose(OC.context_attention(q, k, v.transpose(2, 3), [0, 0], window=1)[0], v)
    assert OC.visible_keys(9, 2, 3) == [0, 1, 7, 8, 9] and OC.visible_keys(9, 0, 0) == list(range(10))


def test_oracle_filters_by_hand():
    z = np.log([0.4, 0.1, 0.2, 0.2, 0.1])
    assert sorted(OS.kept(z, top_k=2)) == [0, 2] and sorted(OS.kept(z, top_k=4)) == [0, 1, 2, 3]
    assert sorted(OS.kept(z, top_p=0.39)) == [0] and sorted(OS.kept(z, top_p=0.59)) == [0, 2] and sorted(OS.kept(z, top_p=0.61)) == [0, 2, 3]
    assert sorted(OS.kept(z, min_p=0.49)) == [0, 2, 3] and sorted(OS.kept(z, temperature=0)) == [0]
    assert sorted(OS.kept(z, top_k=3, top_p=0.74)) == [0, 2]          # of the mass 0.8 that top-k leaves
    w = OS.kept(z)
    assert [OS.draw(w, u)[0] for u in (0.0, 0.3999, 0.41, 0.51, 0.71, 0.95, 1.0)] == [0, 0, 1, 2, 3, 4, 4]
    assert OS.draw(OS.kept(np.full(3, -np.inf)), 0.5)[0] == -1
    T = 2.0
    assert math.isclose(OS.kept(z, temperature=T)[1], (0.1 / 0.4) ** (1 / T))
