"""Serving a batch of images of one prompt: the operators next to the verification step, and the work they are timed on.

Three kinds of case:

  prefix   mulo_attention over a prefix that the sequences of a group share (the conditioning rows of a prompt, and, with
           guidance, those of the empty prompt: two groups) and over the rows that each sequence has of its own.
  window   mulo_attention with a sliding window and sinks: a query sees the first `sinks` rows and the last `window`.
  sample   mulo_sample_filtered: temperature, top-k, top-p and min-p, a draw from given uniforms, and the filtered
           distribution or logits where a drafter or the accept test goes on with them.

Sequence b belongs to group b // (B / G).  Its keys are the S rows of the group's prefix and then its own rows; query j
sits at own row P_b + j, position p = S + P_b + j, and sees key t iff t <= p and (no window, or t < sinks, or
p - t < window).  The cache is libmulo's: keys [.., heads, rows, head_dim], values [.., heads, head_dim, rows].

Sampling orders a row's entries by value, equal ones by index.  The first top_k stay; of those an entry stays if the mass in
front of it is below top_p times the mass of all of them; of those the ones with at least min_p times the largest
probability.  The draw is the first entry, by index, up to which the mass that stays exceeds u times all of it.
"""
import math

import torch

DEV = "cuda:0"
own = False
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases -------------------------------------------------------------------------------------------------------
def _attn(kind, dtype, B, L, nh, nkv, dh, P, G=1, S=0, sinks=0, window=0, ragged=False):
    return dict(kind=kind, dtype=dtype, B=B, L=L, nh=nh, nkv=nkv, dh=dh, P=P, G=G, S=S, sinks=sinks, window=window, ragged=ragged)


def _sample(dtype, R, V, T, k, p, minp, spread, out, cfg=0.0):
    return dict(kind="sample", dtype=dtype, R=R, V=V, T=T, k=k, p=p, minp=minp, spread=spread, out=out, cfg=cfg)


def listed():
    return [
        # a token of eight images of one prompt early in the image: the smallest call, one of 32 a token
        dict(_attn("prefix", "bf16", 8, 1, 32, 32, 128, 100, S=1000), name="prefix_token_8"),
        # a token of 32 images and their unconditional twins, middle of the image: two prefixes, the cache rows themselves
        dict(_attn("prefix", "bf16", 64, 1, 32, 32, 128, 900, G=2, S=2048), name="prefix_token_guided_64"),
        # a row of 16 drafted tokens of 16 variants of one picture, which (64 x 64 tokens and a prompt) is the prefix
        dict(_attn("prefix", "bf16", 16, 16, 32, 32, 128, 330, S=4224), name="prefix_rows_16x16"),
        # the high-resolution block of four images behind a shared prompt: 4096 queries
        dict(_attn("prefix", "bf16", 4, 1024, 32, 32, 128, 2048, S=1024), name="prefix_block_4x1024"),
        # float32 model with shared key heads, sequences of unequal length, ragged prefix
        dict(_attn("prefix", "f32", 6, 5, 16, 4, 64, 300, S=333, ragged=True), name="prefix_f32_6x5"),
        # a token of one image late in a long run: 4 sinks and 500 rows of 8000
        dict(_attn("window", "bf16", 1, 1, 32, 32, 128, 8000, sinks=4, window=500), name="window_token_1"),
        # a token of 32 images, each at its own place: the conditioning rows stay visible, and half of the image
        dict(_attn("window", "bf16", 32, 1, 32, 32, 128, 4223, sinks=128, window=2048, ragged=True), name="window_token_32"),
        # the high-resolution block of four images: the conditioning rows and the last 16 rows of the grid
        dict(_attn("window", "bf16", 4, 1024, 32, 32, 128, 3200, sinks=128, window=1024), name="window_block_4x1024"),
        # one row of 33 tokens of seven sequences, heads of 64 in groups of four, a window that is shorter than a tile
        dict(_attn("window", "bf16", 7, 33, 16, 4, 64, 777, sinks=5, window=50, ragged=True), name="window_rows_7x33"),
        # the next token of one image, the usual setting of such models (top-k 2000 of 16384 codes): latency
        dict(_sample("f32", 1, 16384, 1.0, 2000, 1.0, 0.0, 1.28, "tokens"), name="sample_1"),
        # the next token of 32 guided images: top-k and top-p of the guided logits, the distribution for a later accept test
        dict(_sample("f32", 32, 16384, 0.9, 1000, 0.95, 0.0, 1.0, "tokens+probs", cfg=4.0), name="sample_guided_32"),
        # the target's logits of two drafted blocks, filtered for the accept test
        dict(_sample("f32", 2048, 16384, 1.0, 0, 0.9, 0.001, 2.0, "logits"), name="sample_block_2x1024"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.35:
        R, V = _log(rng, 1, 2048), rng.choice([_log(rng, 500, 150000), 16384, 8192, 1024])
        R = max(1, min(R, 30_000_000 // V))
        cfg = rng.choice([0.0, 0.0, 2.0, 4.0])
        return _sample(rng.choice(["f32", "f32", "bf16"]), R, V, round(rng.uniform(0.5, 1.5), 2), rng.choice([0, 1, 50, V // 8, V // 2]),
                       rng.choice([1.0, round(rng.uniform(0.3, 0.99), 2)]), rng.choice([0.0, 0.0, round(10 ** rng.uniform(-4, -0.7), 4)]),
                       round(rng.uniform(0.8, 3.0), 2), rng.choice(["tokens", "tokens+probs", "logits", "tokens+logits"]), cfg)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    dh = rng.choice([64, 128])
    nkv = rng.choice([4, 8, 16, 32]) if dtype == "bf16" else rng.choice([2, 4, 8])
    nh = nkv * rng.choice([1, 1, 2, 4]) if nkv < 32 else nkv
    L = rng.choice([1, 1, 1, _log(rng, 2, 40), _log(rng, 40, 1024)])
    B = _log(rng, 1, 64 if L < 40 else 4)
    while B * L * nh > (48_000 if dtype == "bf16" else 12_000):
        B, L = max(1, B // 2), max(1, L * 3 // 4)
    P = _log(rng, 1, 4200)
    if rng.random() < 0.5:
        G = 2 if B % 2 == 0 and rng.random() < 0.4 else 1
        c = _attn("prefix", dtype, B, L, nh, nkv, dh, P, G=G, S=_log(rng, 20, 4224), ragged=rng.random() < 0.3)
        if rng.random() < 0.25:          # a window over prefix and own rows
            c.update(sinks=rng.randint(0, 130), window=_log(rng, 16, 2048))
        return c
    return _attn("window", dtype, B, L, nh, nkv, dh, P, sinks=rng.choice([0, 1, 4, rng.randint(5, 300)]), window=_log(rng, 1, 2048),
                 ragged=rng.random() < 0.4)


# ---- what a user's program has in hand -------------------------------------------------------------------------------
def _starts(case, seed):
    """Own rows in front of the block, sequence by sequence: P, or between P / 2 and P."""
    B, P = case["B"], case["P"]
    if not case["ragged"]:
        return [P] * B
    g = torch.Generator().manual_seed(seed + 1)
    return [P] + [int(x) for x in torch.randint(P // 2, P + 1, (B - 1,), generator=g)]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case=case, seed=seed)
    normal = lambda dtype, *shape: torch.empty(*shape, dtype=dtype, device=DEV).normal_(generator=g)
    if case["kind"] == "sample":
        R, V = case["R"], case["V"]
        dt = DTYPES[case["dtype"]]
        z = torch.randn(2 * R if case["cfg"] else R, V, generator=g, device=DEV).mul_(case["spread"])
        if case["cfg"]:     # the twins' logits are near the conditional ones
            z[:R].mul_(0.25).add_(z[R:])
        s["logits"] = z.to(dt)
        s["u"] = torch.rand(R, generator=g, device=DEV)
        s["tokens"] = torch.empty(R, dtype=torch.int32, device=DEV) if "tokens" in case["out"] else None
        s["probs"] = torch.empty(R, V, device=DEV) if "probs" in case["out"] else None
        s["kept"] = torch.empty(R, V, device=DEV) if "logits" in case["out"] else None
        if own:
            import paper_2601_05149_amd as mulo
            s["params"] = mulo.make_sample_params(case["T"], case["k"], case["p"], case["minp"], case["cfg"])
        return s
    dt, B, L, nh, nkv, dh, G, S = DTYPES[case["dtype"]], case["B"], case["L"], case["nh"], case["nkv"], case["dh"], case["G"], case["S"]
    rows, srows = (case["P"] + L + 7) // 8 * 8, (S + 7) // 8 * 8
    # queries and attention output as the projections leave and take them: a token's heads next to each other
    s["q"] = normal(dt, B, L, nh, dh).permute(0, 2, 1, 3)
    s["out"] = torch.empty(B, L, nh, dh, dtype=dt, device=DEV).permute(0, 2, 1, 3)
    s["k"], s["v"] = normal(dt, B, nkv, rows, dh), normal(dt, B, nkv, dh, rows)
    s["pk"], s["pv"] = (normal(dt, G, nkv, srows, dh), normal(dt, G, nkv, dh, srows)) if S else (None, None)
    s["starts"] = _starts(case, seed)
    s["P_seq"] = torch.tensor(s["starts"], dtype=torch.int32, device=DEV) if case["ragged"] else None
    if own:
        import paper_2601_05149_amd as mulo
        s["plan"] = mulo.make_attention(s["q"], s["out"], s["k"], s["v"], case["P"], P_seq=s["P_seq"], prefix_k=s["pk"], prefix_v=s["pv"],
                                        prefix_len=S, sinks=case["sinks"], window=case["window"])
        n = mulo.mulo_attention_workspace_bytes(s["plan"])
        s["work"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------
def _visible(case, starts, j_count, device):
    """Which keys (the prefix's, then the sequence's own, up to the longest) each query sees: [B, L, S + most own rows]."""
    S, n = case["S"], max(starts) + j_count
    pos = S + torch.tensor(starts, device=device)[:, None] + torch.arange(j_count, device=device)[None, :]
    t = torch.arange(S + n, device=device)[None, None, :]
    p = pos[:, :, None]
    see = t <= p
    if case["window"]:
        see = see & ((t < case["sinks"]) | (p - t < case["window"]))
    return see


def _plain_attention(s):
    """Scores against the prefix (once for a group) and against the own rows, one softmax, two products; in float32."""
    case = s["case"]
    B, L, nh, nkv, dh, G, S = case["B"], case["L"], case["nh"], case["nkv"], case["dh"], case["G"], case["S"]
    r, n = nh // nkv * L, max(s["starts"]) + L
    see = _visible(case, s["starts"], L, DEV)
    first = 0
    if case["window"] and not case["sinks"] and not S:      # rows in front of every window are not looked at
        first = max(0, min(s["starts"]) - case["window"] + 1)
    see = see[:, :, first:]
    q = s["q"].float().reshape(B, nkv, r, dh)
    kt = s["k"][:, :, first:n].float().transpose(2, 3).contiguous()
    scores = [torch.matmul(q, kt)]
    if S:
        pkt = s["pk"][:, :, :S].float().transpose(2, 3).contiguous()
        qg = q.reshape(G, B // G, nkv, r, dh).transpose(1, 2).reshape(G, nkv, B // G * r, dh)
        scores.insert(0, torch.matmul(qg, pkt).reshape(G, nkv, B // G, r, S).transpose(1, 2).reshape(B, nkv, r, S))
    z = torch.cat(scores, 3) / math.sqrt(dh)
    z = z.reshape(B, nkv, nh // nkv, L, -1).masked_fill_(~see[:, None, None], -math.inf)
    z = (z - z.amax(-1, keepdim=True)).exp_()
    total = z.sum(-1, keepdim=True)
    z = z.reshape(B, nkv, r, -1)
    o = torch.matmul(z[..., S:], s["v"][:, :, :, first:n].float().transpose(2, 3).contiguous())
    if S:
        zg = z[..., :S].reshape(G, B // G, nkv, r, S).transpose(1, 2).reshape(G, nkv, B // G * r, S)
        og = torch.matmul(zg, s["pv"][:, :, :, :S].float().transpose(2, 3).contiguous())
        o = o + og.reshape(G, nkv, B // G, r, dh).transpose(1, 2).reshape(B, nkv, r, dh)
    return (o.reshape(B, nkv, nh // nkv, L, dh) / total).reshape(B, nh, L, dh).to(s["q"].dtype)


def _row_logits(s):
    """The rows to draw from, float32; guided ones are rounded after every operation, as the accept test takes them."""
    z, R, cfg = s["logits"].float(), s["case"]["R"], s["case"]["cfg"]
    return z[R:] + cfg * (z[:R] - z[R:]) if cfg else z


def _plain_sample(s):
    """Sort, sums in 64 bits (which entries stay, and where a draw lands, are matters of a border), scatter back."""
    case = s["case"]
    z = _row_logits(s)
    R, V = z.shape
    by_value, order = torch.sort(z, dim=1, descending=True, stable=True)
    w = ((by_value.double() - by_value[:, :1].double()) / case["T"]).exp_()
    if 0 < case["k"] < V:
        w[:, case["k"]:] = 0.0
    mass = w.cumsum(1)
    stays = w > 0
    if case["p"] < 1.0:
        stays &= mass - w < case["p"] * mass[:, -1:]
    if case["minp"] > 0.0:
        stays &= w >= case["minp"]
    del mass
    w = torch.zeros_like(w).scatter_(1, order, w * stays)
    stays = torch.zeros_like(stays).scatter_(1, order, stays)
    cum = w.cumsum(1)
    out = []
    if "tokens" in case["out"]:
        out.append((cum <= s["u"].double()[:, None] * cum[:, -1:]).sum(1).to(torch.int32))
    if "probs" in case["out"]:
        out.append((w / cum[:, -1:]).float())
    if "logits" in case["out"]:
        out.append(torch.where(stays, (z.double() / case["T"]).float(), -math.inf))
    return out


def run(s):
    case = s["case"]
    if not own:
        return _plain_sample(s) if case["kind"] == "sample" else _plain_attention(s)
    import paper_2601_05149_amd as mulo
    if case["kind"] == "sample":
        mulo.mulo_sample_filtered(s["params"], s["logits"], s["u"], s["tokens"], s["probs"], s["kept"])
        return [t for t in (s["tokens"], s["probs"], s["kept"]) if t is not None]
    mulo.mulo_attention(s["plan"], s["work"])
    return s["out"]


# ---- the definition, in 64 bits --------------------------------------------------------------------------------------
def _exact_attention(s):
    """Sequence by sequence and head by head of the cache: the keys it sees, laid end to end."""
    case = s["case"]
    B, L, nh, nkv, dh, G, S = case["B"], case["L"], case["nh"], case["nkv"], case["dh"], case["G"], case["S"]
    out = torch.empty(B, nh, L, dh, dtype=torch.float64, device=DEV)
    for b in range(B):
        n, g, P = s["starts"][b] + L, b // (B // G), s["starts"][b]
        p = S + P + torch.arange(L, device=DEV)
        t = torch.arange(S + n, device=DEV)
        hidden = t[None, :] > p[:, None]
        if case["window"]:
            hidden |= (t[None, :] >= case["sinks"]) & (t[None, :] <= p[:, None] - case["window"])
        used = (~hidden).any(0).nonzero()[:, 0]
        k, v = s["k"][b, :, :n].double(), s["v"][b, :, :, :n].double().transpose(1, 2)
        if S:
            k = torch.cat([s["pk"][g, :, :S].double(), k], 1)
            v = torch.cat([s["pv"][g, :, :, :S].double().transpose(1, 2), v], 1)
        k, v, hid = k[:, used], v[:, used], hidden[:, used]
        for h in range(nh):
            kv = h // (nh // nkv)
            a = (s["q"][b, h].double() @ k[kv].T.contiguous()) * dh ** -0.5
            out[b, h] = torch.softmax(a.masked_fill(hid, -math.inf), -1) @ v[kv].contiguous()
    return out


def _exact_sample(s):
    """Row by row: entries fall out of a list that is ordered by a stable sort of the negated values."""
    case = s["case"]
    z32 = _row_logits(s)
    R, V = z32.shape
    tokens, probs, kept = [], [], []
    for i in range(R):
        z = z32[i].double()
        at = torch.argsort(-z, stable=True)
        at = at[:case["k"]] if case["k"] > 0 else at
        e = torch.exp((z[at] - z[at[0]]) / case["T"])
        if case["p"] < 1.0:
            in_front = torch.cat([e.new_zeros(1), torch.cumsum(e, 0)[:-1]])
            n = int(torch.searchsorted(in_front, case["p"] * e.sum()))      # the first that has enough in front of it
            at, e = at[:n], e[:n]
        at = at[e >= case["minp"]].sort()[0]
        e = torch.exp((z[at] - z.max()) / case["T"])
        c = torch.cumsum(e, 0)
        tokens.append(at[torch.searchsorted(c, s["u"][i].double() * c[-1], right=True).clamp_(max=len(at) - 1)])
        if "probs" in case["out"]:
            probs.append(torch.zeros(V, dtype=torch.float64, device=DEV).scatter_(0, at, e / e.sum()))
        if "logits" in case["out"]:
            kept.append(torch.full((V,), -math.inf, dtype=torch.float64, device=DEV).scatter_(0, at, z[at] / case["T"]))
    out = [torch.stack(tokens).to(torch.int32)] if "tokens" in case["out"] else []
    return out + [torch.stack(x) for x in (probs, kept) if x]


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_sample(s) if case["kind"] == "sample" else _exact_attention(s)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "sample":
        e = 2 if case["dtype"] == "bf16" else 4
        R, V = case["R"], case["V"]
        written = 4 * R * ("tokens" in case["out"]) + 4 * R * V * (("probs" in case["out"]) + ("logits" in case["out"]))
        return dict(bytes=float(e * R * V * (2 if case["cfg"] else 1) + 4 * R + written), flops=0.0)
    B, L, nh, nkv, dh, G, S = case["B"], case["L"], case["nh"], case["nkv"], case["dh"], case["G"], case["S"]
    e = 2 if case["dtype"] == "bf16" else 4
    starts = [case["P"] * (0.75 if case["ragged"] and b else 1.0) for b in range(B)]      # on average
    win, sinks = case["window"], case["sinks"]
    pairs = own_rows = 0.0
    shared = [0.0] * G
    for b, P in enumerate(starts):
        first, last = S + P, S + P + L - 1                  # positions of the block
        if not win:
            pairs += L * (first + last) / 2 + L
            own_rows += P + L
            shared[b // (B // G)] = S
            continue
        pairs += L * min(first + (L + 1) / 2, win + min(sinks, max(0, first - win)))
        lo = max(0, first - win + 1)                        # the window of the first query, and the sinks in front of it
        own_rows += last + 1 - max(lo, S) + max(0, min(sinks, lo) - S)
        shared[b // (B // G)] = max(shared[b // (B // G)], max(0, S - lo) + min(sinks, S, lo))
    return dict(bytes=float(e * dh * (2 * B * L * nh + 2 * nkv * (own_rows + sum(shared)))), flops=4.0 * dh * nh * pairs)
