"""ctypes binding of libmulo: the same entry points as include/mulo.h, taking
torch tensors (device memory) and marshalling them to plain pointers.  No
computation happens here, and there is no fallback: if the library is missing
or a call fails, an exception is raised.
"""
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmulo.so")

MULO_OK = 0
MULO_F32, MULO_BF16 = 0, 1
STATUS_NAMES = {0: "MULO_OK", 1: "MULO_ERR_NULL", 2: "MULO_ERR_SHAPE", 3: "MULO_ERR_RANGE",
                4: "MULO_ERR_ALLOC", 5: "MULO_ERR_HIP", 6: "MULO_ERR_UNSUPPORTED"}
EXPORTS = ["mulo_status_string", "mulo_check_model_cfg", "mulo_check_step_params", "mulo_workspace_bytes",
           "mulo_create", "mulo_destroy", "mulo_upsample_draft", "mulo_verify_forward",
           "mulo_accept_local_resample", "mulo_accept_local_resample_static", "mulo_verify_step", "mulo_resample_sequential", "mulo_rejection_islands", "mulo_resample_islands", "mulo_workspace_read", "mulo_profile",
           "mulo_profile_read", "mulo_check_attention", "mulo_attention_workspace_bytes", "mulo_attention",
           "mulo_attach_prefix", "mulo_set_window", "mulo_sample_filtered",
           "mulo_packed_tile_bytes", "mulo_check_packed_rows", "mulo_pack_rows", "mulo_unpack_rows", "mulo_check_packed_attention",
           "mulo_packed_attention_workspace_bytes", "mulo_packed_attention"]


class MuloError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s failed: %s (%s)" % (where, STATUS_NAMES.get(status, status), status_string(status)))


class ModelCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "head_dim", "d_ffn", "vocab",
                                         "max_batch", "max_seq", "max_block", "dtype")] + [("rms_eps", C.c_float),
                                                                                             ("stream_copy", C.c_int32)]


class Weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("embed", "attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate",
                                          "w_up", "w_down", "final_norm", "lm_head", "rope_cos", "rope_sin")]


class KV(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p)]


class StepParams(C.Structure):
    _fields_ = [("H", C.c_int32), ("W", C.c_int32), ("n0", C.c_int32), ("L", C.c_int32),
                ("radius", C.c_int32), ("expand", C.c_int32), ("pool_k", C.c_int32),
                ("nbr", C.c_void_p), ("resample_mode", C.c_int32),
                ("seed", C.c_uint64), ("rng_counter", C.c_uint64),
                ("accept_mode", C.c_int32), ("tau", C.c_float), ("cfg_scale", C.c_float)]


class AttentionArgs(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("dtype", "B", "L", "n_heads", "n_kv_heads", "head_dim")] + [("q", C.c_void_p)] +
                [(n, C.c_int64) for n in ("q_batch", "q_head", "q_row")] + [("out", C.c_void_p)] +
                [(n, C.c_int64) for n in ("out_batch", "out_head", "out_row")] + [("k", C.c_void_p), ("v", C.c_void_p)] +
                [(n, C.c_int64) for n in ("k_batch", "k_head", "k_row", "v_batch", "v_head", "v_chan")] +
                [("rows", C.c_int32), ("P", C.c_int32), ("P_seq", C.c_void_p), ("prefix_k", C.c_void_p), ("prefix_v", C.c_void_p)] +
                [(n, C.c_int64) for n in ("prefix_k_group", "prefix_k_head", "prefix_k_row", "prefix_v_group", "prefix_v_head",
                                          "prefix_v_chan")] +
                [(n, C.c_int32) for n in ("n_prefix", "prefix_len", "prefix_rows", "sinks", "window")] + [("scale", C.c_float)])


class PackedKV(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("format", "B", "n_kv_heads", "head_dim", "rows")] + [(n, C.c_void_p) for n in ("k", "v")] +
                [(n, C.c_int64) for n in ("batch", "head")])


class KVRows(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("dtype", "L")] + [(n, C.c_void_p) for n in ("k", "v")] +
                [(n, C.c_int64) for n in ("k_batch", "k_head", "k_row", "v_batch", "v_head", "v_row", "v_chan")] +
                [("P", C.c_int32), ("P_seq", C.c_void_p)])


class PackedAttentionArgs(C.Structure):
    _fields_ = ([("kv", PackedKV)] + [(n, C.c_int32) for n in ("dtype", "L", "n_heads")] + [("q", C.c_void_p)] +
                [(n, C.c_int64) for n in ("q_batch", "q_head", "q_row")] + [("out", C.c_void_p)] +
                [(n, C.c_int64) for n in ("out_batch", "out_head", "out_row")] +
                [("P", C.c_int32), ("P_seq", C.c_void_p), ("sinks", C.c_int32), ("window", C.c_int32), ("scale", C.c_float)])


class Prefix(C.Structure):
    _fields_ = ([("kv", KV)] + [(n, C.c_int32) for n in ("n_prefix", "max_prefix", "rows", "len")] +
                [("rope_cos", C.c_void_p), ("rope_sin", C.c_void_p)])


class SampleParams(C.Structure):
    _fields_ = [("temperature", C.c_double), ("top_p", C.c_double), ("min_p", C.c_double), ("top_k", C.c_int32),
                ("cfg_scale", C.c_float)]


_lib = None


def load_library():
    """dlopen libmulo.so (built in-tree by paper_2601_05149_amd/build.py); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libmulo.so is not built: run `python -m paper_2601_05149_amd.build` "
                          "(or __graft_entry__.build()) first; there is no fallback path")
    lib = C.CDLL(LIB_PATH)
    P, I32, I64 = C.c_void_p, C.c_int32, C.c_int64
    lib.mulo_status_string.restype = C.c_char_p
    lib.mulo_status_string.argtypes = [C.c_int]
    lib.mulo_check_model_cfg.argtypes = [C.POINTER(ModelCfg)]
    lib.mulo_check_step_params.argtypes = [C.POINTER(ModelCfg), I32, C.POINTER(StepParams)]
    lib.mulo_workspace_bytes.restype = C.c_uint64
    lib.mulo_workspace_bytes.argtypes = [C.POINTER(ModelCfg)]
    lib.mulo_create.argtypes = [C.POINTER(ModelCfg), C.POINTER(Weights), P, C.POINTER(P)]
    lib.mulo_destroy.restype = None
    lib.mulo_destroy.argtypes = [P]
    lib.mulo_upsample_draft.argtypes = [P, I32, I32, I32, I32, P, I32, P, P, P, P, P]
    lib.mulo_verify_forward.argtypes = [P, C.POINTER(KV), I32, I32, I32, P, P, P]
    lib.mulo_accept_local_resample.argtypes = [P, I32, C.POINTER(StepParams), P, P, P, I64, P, P, P, P, P, P, P]
    lib.mulo_accept_local_resample_static.argtypes = [P, I32, I32, C.POINTER(StepParams), P, P, P, I64, P, P, P, P, P, P, P]
    lib.mulo_verify_step.argtypes = [P, C.POINTER(KV), I32, I32, C.POINTER(StepParams), I32, I32, I32, P, I32,
                                     P, P, P, P, P, P, P, P, P]
    lib.mulo_resample_sequential.argtypes = [P, C.POINTER(KV), I32, I32, I32, I32, C.c_uint64, C.c_uint64, P, P, P, P]
    lib.mulo_rejection_islands.argtypes = [P, I32, I32, I32, I32, P, P, P, P]
    lib.mulo_resample_islands.argtypes = [P, C.POINTER(KV), I32, I32, I32, I32, I32, C.c_uint64, C.c_uint64, P, P, P, P, P, P]
    lib.mulo_workspace_read.argtypes = [P, I32, P, C.c_uint64]
    lib.mulo_profile.argtypes = [P, I32]
    lib.mulo_profile_read.argtypes = [P, C.POINTER(C.c_float), C.POINTER(I32)]
    lib.mulo_check_attention.argtypes = [C.POINTER(AttentionArgs)]
    lib.mulo_attention_workspace_bytes.restype = C.c_uint64
    lib.mulo_attention_workspace_bytes.argtypes = [C.POINTER(AttentionArgs)]
    lib.mulo_attention.argtypes = [P, C.POINTER(AttentionArgs), P, C.c_uint64]
    lib.mulo_attach_prefix.argtypes = [P, C.POINTER(Prefix)]
    lib.mulo_set_window.argtypes = [P, I32, I32]
    lib.mulo_sample_filtered.argtypes = [P, C.POINTER(SampleParams), I32, I32, I32, P, I64, P, P, P, P]
    lib.mulo_packed_tile_bytes.restype = C.c_uint64
    lib.mulo_packed_tile_bytes.argtypes = [I32, I32]
    lib.mulo_check_packed_rows.argtypes = [C.POINTER(PackedKV), C.POINTER(KVRows)]
    lib.mulo_pack_rows.argtypes = lib.mulo_unpack_rows.argtypes = [P, C.POINTER(PackedKV), C.POINTER(KVRows)]
    lib.mulo_check_packed_attention.argtypes = [C.POINTER(PackedAttentionArgs)]
    lib.mulo_packed_attention_workspace_bytes.restype = C.c_uint64
    lib.mulo_packed_attention_workspace_bytes.argtypes = [C.POINTER(PackedAttentionArgs)]
    lib.mulo_packed_attention.argtypes = [P, C.POINTER(PackedAttentionArgs), P, C.c_uint64]
    for n in EXPORTS:
        if n not in ("mulo_status_string", "mulo_workspace_bytes", "mulo_destroy", "mulo_attention_workspace_bytes",
                     "mulo_packed_tile_bytes", "mulo_packed_attention_workspace_bytes"):
            getattr(lib, n).restype = C.c_int
    _lib = lib
    return lib


def status_string(status):
    return load_library().mulo_status_string(int(status)).decode()


def _ptr(t, dtype=None, allow_none=False):
    if t is None:
        if allow_none:
            return None
        raise ValueError("required tensor is None")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("libmulo takes contiguous device tensors")
    if dtype is not None and t.dtype != dtype:
        raise ValueError("expected %s, got %s" % (dtype, t.dtype))
    return t.data_ptr()


def _check(status, where):
    if status != MULO_OK:
        raise MuloError(status, where)


def make_cfg(model, max_batch, max_seq, max_block, stream_copy=False):
    bf16 = model["dtype"] == "bf16"
    return ModelCfg(model["n_layers"], model["d_model"], model["n_heads"], model["head_dim"], model["d_ffn"],
                    model["vocab"], max_batch, max_seq, max_block,
                    MULO_BF16 if bf16 else MULO_F32, model.get("rms_eps", 1e-5), 1 if (stream_copy and bf16) else 0)


MULO_ACCEPT_RATIO, MULO_ACCEPT_TAU = 0, 1


def make_params(H, W, n0, L, radius, expand=1, pool_k=1, nbr=None, resample_mode=0, seed=0, rng_counter=0,
                accept_mode=MULO_ACCEPT_RATIO, tau=0.0, cfg_scale=0.0):
    return StepParams(H, W, n0, L, radius, expand, pool_k, _ptr(nbr, torch.int32, True), resample_mode,
                      seed, rng_counter, accept_mode, tau, cfg_scale)


class Ctx:
    """Owns a mulo_ctx* and keeps the weight tensors alive (the library borrows them)."""

    def __init__(self, handle, cfg, keep):
        self.handle, self.cfg, self._keep = handle, cfg, keep
        self.tdtype = torch.bfloat16 if cfg.dtype == MULO_BF16 else torch.float32

    def __del__(self):
        try:
            mulo_destroy(self)
        except Exception:
            pass


def mulo_create(cfg, weights, rope_cos, rope_sin, stream=None):
    """weights: dict of device tensors (see mulo_weights); returns Ctx."""
    lib = load_library()
    tdt = torch.bfloat16 if cfg.dtype == MULO_BF16 else torch.float32
    names = ["embed", "attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down",
             "final_norm", "lm_head"]
    w = Weights(*[_ptr(weights[n], tdt) for n in names], _ptr(rope_cos, torch.float32), _ptr(rope_sin, torch.float32))
    st = torch.cuda.current_stream().cuda_stream if stream is None else stream
    out = C.c_void_p()
    _check(lib.mulo_create(C.byref(cfg), C.byref(w), C.c_void_p(st), C.byref(out)), "mulo_create")
    return Ctx(out, cfg, [weights, rope_cos, rope_sin])


def mulo_destroy(ctx):
    if ctx is not None and ctx.handle:
        load_library().mulo_destroy(ctx.handle)
        ctx.handle = None


def alloc_kv(ctx, device="cuda", zero=True):
    """Allocate the KV cache in the layout mulo_kv documents; returns (k, v) tensors."""
    c = ctx.cfg
    mk = torch.zeros if zero else torch.empty
    k = mk(c.n_layers, c.max_batch, c.n_heads, c.max_seq, c.head_dim, dtype=ctx.tdtype, device=device)
    v = mk(c.n_layers, c.max_batch, c.n_heads, c.head_dim, c.max_seq, dtype=ctx.tdtype, device=device)
    return k, v


def mulo_upsample_draft(ctx, B, h, w, r, draft, input_is_probs, draft_tokens, tokens_hi, q_lo, q_row, q_hi=None):
    f32, i32 = torch.float32, torch.int32
    _check(load_library().mulo_upsample_draft(
        ctx.handle, B, h, w, r, _ptr(draft, f32), int(input_is_probs), _ptr(draft_tokens, i32),
        _ptr(tokens_hi, i32), _ptr(q_lo, f32), _ptr(q_row, i32), _ptr(q_hi, f32, True)), "mulo_upsample_draft")


def mulo_verify_forward(ctx, kv, B, L, P, in_tokens, in_embeds, logits):
    kvs = KV(_ptr(kv[0], ctx.tdtype), _ptr(kv[1], ctx.tdtype))
    _check(load_library().mulo_verify_forward(
        ctx.handle, C.byref(kvs), B, L, P, _ptr(in_tokens, torch.int32, True), _ptr(in_embeds, ctx.tdtype, True),
        _ptr(logits, torch.float32)), "mulo_verify_forward")


def mulo_accept_local_resample(ctx, B, params, logits, q, q_row, q_batch_stride, draft_tokens, tokens_out,
                               accept, mask, t0, stats, p_probs=None):
    f32, i32, u8 = torch.float32, torch.int32, torch.uint8
    _check(load_library().mulo_accept_local_resample(
        ctx.handle, B, C.byref(params), _ptr(logits, f32), _ptr(q, f32, True), _ptr(q_row, i32, True),
        int(q_batch_stride), _ptr(draft_tokens, i32), _ptr(tokens_out, i32), _ptr(accept, u8), _ptr(mask, u8),
        _ptr(t0, i32), _ptr(stats, i32), _ptr(p_probs, f32, True)), "mulo_accept_local_resample")


MULO_STATIC_MAX_ROWS = 65536


def mulo_accept_local_resample_static(vocab, B, params, logits, q, q_row, q_batch_stride, draft_tokens, tokens_out,
                                      accept, mask, t0, stats, p_probs=None, stream=None):
    """The decision stage without a context (allocates nothing); stream: a raw hipStream_t or None for
    torch's current stream."""
    f32, i32, u8 = torch.float32, torch.int32, torch.uint8
    st = torch.cuda.current_stream().cuda_stream if stream is None else stream
    _check(load_library().mulo_accept_local_resample_static(
        C.c_void_p(st), vocab, B, C.byref(params), _ptr(logits, f32), _ptr(q, f32, True), _ptr(q_row, i32, True),
        int(q_batch_stride), _ptr(draft_tokens, i32), _ptr(tokens_out, i32), _ptr(accept, u8), _ptr(mask, u8),
        _ptr(t0, i32), _ptr(stats, i32), _ptr(p_probs, f32, True)), "mulo_accept_local_resample_static")


def mulo_verify_step(ctx, kv, B, P, params, h_blk, w, r, draft, input_is_probs, draft_tokens, prev_tokens,
                     tokens_out, accept, mask, t0, stats, tokens_hi=None, logits=None):
    f32, i32, u8 = torch.float32, torch.int32, torch.uint8
    kvs = KV(_ptr(kv[0], ctx.tdtype), _ptr(kv[1], ctx.tdtype))
    _check(load_library().mulo_verify_step(
        ctx.handle, C.byref(kvs), B, P, C.byref(params), h_blk, w, r, _ptr(draft, f32, True), int(input_is_probs),
        _ptr(draft_tokens, i32), _ptr(prev_tokens, i32), _ptr(tokens_out, i32), _ptr(accept, u8),
        _ptr(mask, u8), _ptr(t0, i32), _ptr(stats, i32), _ptr(tokens_hi, i32, True), _ptr(logits, f32, True)),
        "mulo_verify_step")


def mulo_resample_sequential(ctx, kv, B, P, L, u_start, seed, rng_counter, prev_tokens, mask, tokens, logits=None):
    f32, i32, u8 = torch.float32, torch.int32, torch.uint8
    kvs = KV(_ptr(kv[0], ctx.tdtype), _ptr(kv[1], ctx.tdtype))
    _check(load_library().mulo_resample_sequential(
        ctx.handle, C.byref(kvs), B, P, L, u_start, C.c_uint64(seed), C.c_uint64(rng_counter), _ptr(prev_tokens, i32),
        _ptr(mask, u8), _ptr(tokens, i32), _ptr(logits, f32, True)), "mulo_resample_sequential")


def mulo_rejection_islands(ctx, B, W, n0, L, mask, island, rank, counts):
    i32, u8 = torch.int32, torch.uint8
    _check(load_library().mulo_rejection_islands(ctx.handle, B, W, n0, L, _ptr(mask, u8), _ptr(island, i32), _ptr(rank, i32),
                                                 _ptr(counts, i32)), "mulo_rejection_islands")


def mulo_resample_islands(ctx, kv, B, P, L, n_passes, max_islands, seed, rng_counter, prev_tokens, mask, rank, tokens,
                          logits=None, overflow=None):
    f32, i32, u8 = torch.float32, torch.int32, torch.uint8
    kvs = KV(_ptr(kv[0], ctx.tdtype), _ptr(kv[1], ctx.tdtype))
    _check(load_library().mulo_resample_islands(
        ctx.handle, C.byref(kvs), B, P, L, n_passes, max_islands, C.c_uint64(seed), C.c_uint64(rng_counter),
        _ptr(prev_tokens, i32), _ptr(mask, u8), _ptr(rank, i32), _ptr(tokens, i32), _ptr(logits, f32, True),
        _ptr(overflow, i32, True)), "mulo_resample_islands")


MULO_WS_RESIDUAL, MULO_WS_NORMED, MULO_WS_Q, MULO_WS_ATTN, MULO_WS_FFN = range(5)


def mulo_workspace_read(ctx, which, dst):
    """Copy a workspace buffer of the last forward pass into the (contiguous, device) tensor dst."""
    _check(load_library().mulo_workspace_read(ctx.handle, which, _ptr(dst), dst.numel() * dst.element_size()),
           "mulo_workspace_read")


def _strided(t, dtype, name, dims):
    """Pointer and strides (elements; 0 where there is only one) of a tensor whose last dimension is contiguous."""
    if t.dim() != dims or not t.is_cuda or t.dtype != dtype or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError("%s: expected a device tensor of %d dimensions, %s, contiguous in the last" % (name, dims, dtype))
    return t.data_ptr(), [t.stride(i) if t.shape[i] > 1 else 0 for i in range(dims - 1)]


def _on_device(device, stream, call):
    """Runs a call without a context on its tensors' device; stream: a raw hipStream_t, or torch's current stream of that device."""
    st = torch._C._cuda_getCurrentRawStream(device.index) if stream is None else stream
    if torch._C._cuda_getDevice() == device.index:
        return call(st)
    with torch.cuda.device(device):
        return call(st)


class Attention:
    """Arguments of mulo_attention, checked, with the tensors they point into."""

    def __init__(self, args, keep, device):
        self.args, self._keep, self.device = args, keep, device
        self.ref = C.byref(args)


def make_attention(q, out, k, v, P, P_seq=None, prefix_k=None, prefix_v=None, prefix_len=0, sinks=0, window=0, scale=0.0):
    """q, out [B, n_heads, L, head_dim]; k [B, n_kv_heads, rows, head_dim]; v [B, n_kv_heads, head_dim, rows]; P_seq int32 [B]
    or None; prefix_k [groups, n_kv_heads, prefix_rows, head_dim], prefix_v [groups, n_kv_heads, head_dim, prefix_rows]: any
    strides with a contiguous last dimension."""
    if q.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("expected bfloat16 or float32, got %s" % q.dtype)
    B, nh, L, dh = q.shape
    nkv, rows = k.shape[1], k.shape[2]
    if out.shape != q.shape or k.shape != (B, nkv, rows, dh) or v.shape != (B, nkv, dh, rows):
        raise ValueError("q, out, k and v do not fit together")
    tensors = [q, out, k, v]
    a = AttentionArgs(dtype=MULO_BF16 if q.dtype == torch.bfloat16 else MULO_F32, B=B, L=L, n_heads=nh, n_kv_heads=nkv, head_dim=dh,
                      rows=rows, P=P, n_prefix=1, prefix_len=prefix_len, sinks=sinks, window=window, scale=scale)
    a.q, (a.q_batch, a.q_head, a.q_row) = _strided(q, q.dtype, "q", 4)
    a.out, (a.out_batch, a.out_head, a.out_row) = _strided(out, q.dtype, "out", 4)
    a.k, (a.k_batch, a.k_head, a.k_row) = _strided(k, q.dtype, "k", 4)
    a.v, (a.v_batch, a.v_head, a.v_chan) = _strided(v, q.dtype, "v", 4)
    if P_seq is not None:
        if P_seq.shape != (B,):
            raise ValueError("P_seq has one entry per sequence")
        a.P_seq = _ptr(P_seq, torch.int32)
        tensors.append(P_seq)
    if prefix_len and (prefix_k is None or prefix_v is None):
        raise ValueError("a prefix of %d rows without its keys or values" % prefix_len)
    if prefix_len:
        G, prows = prefix_k.shape[0], prefix_k.shape[2]
        if prefix_k.shape != (G, nkv, prows, dh) or prefix_v.shape != (G, nkv, dh, prows):
            raise ValueError("the prefix does not fit the cache")
        a.n_prefix, a.prefix_rows = G, prows
        a.prefix_k, (a.prefix_k_group, a.prefix_k_head, a.prefix_k_row) = _strided(prefix_k, q.dtype, "prefix_k", 4)
        a.prefix_v, (a.prefix_v_group, a.prefix_v_head, a.prefix_v_chan) = _strided(prefix_v, q.dtype, "prefix_v", 4)
        tensors += [prefix_k, prefix_v]
    if any(t.device != q.device for t in tensors):
        raise ValueError("the tensors of a call lie on one device")
    _check(load_library().mulo_check_attention(C.byref(a)), "mulo_check_attention")
    return Attention(a, tensors, q.device)


def mulo_attention_workspace_bytes(attention):
    with torch.cuda.device(attention.device):
        return load_library().mulo_attention_workspace_bytes(attention.ref)


def mulo_attention(attention, workspace=None, stream=None):
    """Writes `out` of make_attention; workspace: a contiguous device tensor or None."""
    ptr, n = (None, 0) if workspace is None else (_ptr(workspace), workspace.numel() * workspace.element_size())
    if workspace is not None and workspace.device != attention.device:
        raise ValueError("the workspace lies on another device")
    lib = load_library()
    _check(_on_device(attention.device, stream, lambda st: lib.mulo_attention(st, attention.ref, ptr, n)), "mulo_attention")


def mulo_attach_prefix(ctx, kv=None, length=0, rope_cos=None, rope_sin=None, n_prefix=None):
    """kv: the (k, v) tensors of a cache whose max_batch sequences are the prefixes (alloc_kv of the context that made them);
    rope_cos, rope_sin: float32 [max_seq, head_dim / 2] of ctx, row i for position length + i.  kv None detaches."""
    if kv is None:
        _check(load_library().mulo_attach_prefix(ctx.handle, None), "mulo_attach_prefix")
        ctx._prefix = None
        return
    c = ctx.cfg
    k, v = kv
    n, rows = k.shape[1], k.shape[3]
    if k.shape != (c.n_layers, n, c.n_heads, rows, c.head_dim) or v.shape != (c.n_layers, n, c.n_heads, c.head_dim, rows):
        raise ValueError("the prefix is not a cache of this model")
    if any(t is None or t.shape != (c.max_seq, c.head_dim // 2) for t in (rope_cos, rope_sin)):
        raise ValueError("the rotary tables of the prefix have a row for every cache row of the context")
    p = Prefix(KV(_ptr(k, ctx.tdtype), _ptr(v, ctx.tdtype)), n if n_prefix is None else n_prefix, n, rows, length,
               _ptr(rope_cos, torch.float32), _ptr(rope_sin, torch.float32))
    _check(load_library().mulo_attach_prefix(ctx.handle, C.byref(p)), "mulo_attach_prefix")
    ctx._prefix = [k, v, rope_cos, rope_sin]


def mulo_set_window(ctx, sinks, window):
    _check(load_library().mulo_set_window(ctx.handle, sinks, window), "mulo_set_window")


def make_sample_params(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, cfg_scale=0.0):
    return SampleParams(temperature, top_p, min_p, top_k, cfg_scale)


def mulo_sample_filtered(params, logits, u=None, tokens=None, probs=None, logits_out=None, stream=None):
    """logits [rows, vocab] (2 rows conditional, then unconditional, with params.cfg_scale), float32 or bfloat16, rows at any
    stride; u float32 [rows]; tokens int32 [rows], probs and logits_out float32 [rows, vocab], each or None."""
    if logits.dim() != 2 or logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("logits: expected a matrix of float32 or bfloat16")
    ptr, (stride,) = _strided(logits, logits.dtype, "logits", 2)
    n, V = logits.shape
    rows = n // 2 if params.cfg_scale > 0 else n
    if params.cfg_scale > 0 and n % 2:
        raise ValueError("guidance takes a conditional and an unconditional row each")
    f32, i32 = torch.float32, torch.int32
    device, lib = logits.device, load_library()

    def ptr_of(t, dtype, *shape):
        if t is None:
            return None
        if t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
            raise ValueError("expected %s, contiguous, %s on the logits' device" % (shape, dtype))
        return t.data_ptr()

    u, tokens = ptr_of(u, f32, rows), ptr_of(tokens, i32, rows)
    probs, out = ptr_of(probs, f32, rows, V), ptr_of(logits_out, f32, rows, V)
    _check(_on_device(device, stream, lambda st: lib.mulo_sample_filtered(
        st, C.byref(params), rows, V, MULO_BF16 if logits.dtype == torch.bfloat16 else MULO_F32, ptr, stride if n > 1 else V,
        u, tokens, probs, out)), "mulo_sample_filtered")


MULO_FP4, MULO_FP8 = 0, 1


class Packed:
    """A packed cache: the tensors of its tiles and the struct that points to them."""

    def __init__(self, args, k, v):
        self.args, self.k, self.v, self.device = args, k, v, k.device
        self.ref = C.byref(args)


def mulo_packed_tile_bytes(format, head_dim):
    return load_library().mulo_packed_tile_bytes(format, head_dim)


def make_packed_kv(k, v, format, head_dim):
    """k, v uint8 [B, n_kv_heads, rows / 64, mulo_packed_tile_bytes], the last two dimensions contiguous, strides alike."""
    size = mulo_packed_tile_bytes(format, head_dim)
    if not size:
        raise ValueError("no packed cache of format %s with heads of %s" % (format, head_dim))
    for t in (k, v):
        if t.dim() != 4 or not t.is_cuda or t.dtype != torch.uint8 or t.shape[3] != size or t.stride(3) != 1 or (t.shape[2] > 1 and t.stride(2) != size):
            raise ValueError("expected tiles, a device tensor [B, heads, tiles, %d] of uint8, contiguous in the last two dimensions" % size)
    if k.shape != v.shape or k.device != v.device:
        raise ValueError("keys and values do not fit together")
    strides = [[t.stride(i) if t.shape[i] > 1 else 0 for i in range(2)] for t in (k, v)]
    if strides[0] != strides[1]:
        raise ValueError("keys and values have the same strides")
    B, nkv, tiles = k.shape[:3]
    return Packed(PackedKV(format, B, nkv, head_dim, tiles * 64, k.data_ptr(), v.data_ptr(), *strides[0]), k, v)


def alloc_packed_kv(B, n_kv_heads, rows, head_dim, format=MULO_FP4, device="cuda"):
    """A packed cache of at least `rows` rows (whole tiles of 64) a sequence, zeros."""
    size = mulo_packed_tile_bytes(format, head_dim)
    k, v = (torch.zeros(B, n_kv_heads, (rows + 63) // 64, size, dtype=torch.uint8, device=device) for _ in range(2))
    return make_packed_kv(k, v, format, head_dim)


class Rows:
    """Rows of numbers of a packed cache's sequences, with the tensors they point into."""

    def __init__(self, args, keep, shape, device):
        self.args, self._keep, self.shape, self.device = args, keep, shape, device
        self.ref = C.byref(args)


def make_kv_rows(k, v, P, P_seq=None):
    """k, v [B, n_kv_heads, L, head_dim], each or None: k in any strides with a contiguous last dimension, v also with a contiguous
    third one (a mulo_kv's values, transposed); P_seq int32 [B] or None."""
    given = [t for t in (k, v) if t is not None]
    if not given or any(t.dim() != 4 or t.shape != given[0].shape or t.dtype != given[0].dtype or t.device != given[0].device for t in given):
        raise ValueError("k and v do not fit together")
    dtype, (B, nkv, L, dh) = given[0].dtype, given[0].shape
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("expected bfloat16 or float32, got %s" % dtype)
    r = KVRows(dtype=MULO_BF16 if dtype == torch.bfloat16 else MULO_F32, L=L, P=P)
    if k is not None:
        r.k, (r.k_batch, r.k_head, r.k_row) = _strided(k, dtype, "k", 4)
    if v is not None:
        if not v.is_cuda or (v.stride(3) != 1 and L > 1 and v.stride(2) != 1):
            raise ValueError("v: expected a device tensor, contiguous in its rows or in its channels")
        r.v = v.data_ptr()
        r.v_batch, r.v_head, r.v_row = (v.stride(i) if v.shape[i] > 1 else 0 for i in range(3))
        r.v_chan = v.stride(3)
    keep = given
    if P_seq is not None:
        if P_seq.shape != (B,) or P_seq.device != given[0].device:
            raise ValueError("P_seq has one entry per sequence, on the device of the rows")
        r.P_seq = _ptr(P_seq, torch.int32)
        keep = given + [P_seq]
    return Rows(r, keep, (B, nkv, dh), given[0].device)


def _packed_rows(name, packed, rows, stream):
    if rows.shape != (packed.args.B, packed.args.n_kv_heads, packed.args.head_dim) or rows.device != packed.device:
        raise ValueError("the rows are not those of this cache")
    call = getattr(load_library(), name)
    _check(_on_device(packed.device, stream, lambda st: call(st, packed.ref, rows.ref)), name)


def mulo_pack_rows(packed, rows, stream=None):
    """Writes the rows of make_kv_rows into the cache of make_packed_kv."""
    _packed_rows("mulo_pack_rows", packed, rows, stream)


def mulo_unpack_rows(packed, rows, stream=None):
    """Writes rows of the cache into the tensors of make_kv_rows."""
    _packed_rows("mulo_unpack_rows", packed, rows, stream)


class PackedAttention:
    """Arguments of mulo_packed_attention, checked, with the tensors they point into."""

    def __init__(self, args, keep, device):
        self.args, self._keep, self.device = args, keep, device
        self.ref = C.byref(args)


def make_packed_attention(packed, q, out, P, P_seq=None, sinks=0, window=0, scale=0.0):
    """q, out [B, n_heads, L, head_dim], any strides with a contiguous last dimension; P_seq int32 [B] or None."""
    if q.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("expected bfloat16 or float32, got %s" % q.dtype)
    B, nh, L, dh = q.shape
    if out.shape != q.shape or (B, dh) != (packed.args.B, packed.args.head_dim):
        raise ValueError("q, out and the cache do not fit together")
    a = PackedAttentionArgs(kv=packed.args, dtype=MULO_BF16 if q.dtype == torch.bfloat16 else MULO_F32, L=L, n_heads=nh, P=P, sinks=sinks,
                            window=window, scale=scale)
    a.q, (a.q_batch, a.q_head, a.q_row) = _strided(q, q.dtype, "q", 4)
    a.out, (a.out_batch, a.out_head, a.out_row) = _strided(out, q.dtype, "out", 4)
    tensors = [q, out, packed.k, packed.v]
    if P_seq is not None:
        if P_seq.shape != (B,):
            raise ValueError("P_seq has one entry per sequence")
        a.P_seq = _ptr(P_seq, torch.int32)
        tensors.append(P_seq)
    if any(t.device != q.device for t in tensors):
        raise ValueError("the tensors of a call lie on one device")
    _check(load_library().mulo_check_packed_attention(C.byref(a)), "mulo_check_packed_attention")
    return PackedAttention(a, tensors, q.device)


def mulo_packed_attention_workspace_bytes(attention):
    with torch.cuda.device(attention.device):
        return load_library().mulo_packed_attention_workspace_bytes(attention.ref)


def mulo_packed_attention(attention, workspace=None, stream=None):
    """Writes `out` of make_packed_attention; workspace: a contiguous device tensor or None."""
    ptr, n = (None, 0) if workspace is None else (_ptr(workspace), workspace.numel() * workspace.element_size())
    if workspace is not None and workspace.device != attention.device:
        raise ValueError("the workspace lies on another device")
    lib = load_library()
    _check(_on_device(attention.device, stream, lambda st: lib.mulo_packed_attention(st, attention.ref, ptr, n)), "mulo_packed_attention")


PROF_CLASSES = ["gemm_qkv", "gemm_out", "gemm_gate_up", "gemm_down", "gemm_lm_head", "attention", "norm_embed",
                "upsample", "accept", "mask_sample", "other"]


def mulo_profile(ctx, enable):
    _check(load_library().mulo_profile(ctx.handle, int(enable)), "mulo_profile")


def mulo_profile_read(ctx):
    """Returns {class name: (milliseconds, launches)} accumulated since the last read."""
    n = len(PROF_CLASSES)
    ms, cnt = (C.c_float * n)(), (C.c_int32 * n)()
    _check(load_library().mulo_profile_read(ctx.handle, ms, cnt), "mulo_profile_read")
    return {PROF_CLASSES[i]: (float(ms[i]), int(cnt[i])) for i in range(n)}
