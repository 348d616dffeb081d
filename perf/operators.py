"""Operators of a serving batch whose sequences have lengths and pages of their own: what is timed, and their plain forms.

Four kinds of work, at the sizes a server of this library's layers calls them with:

    attention  rt_paged_attention: one new token per sequence over a paged key-value cache
    cache      rt_cache_write, rt_cache_read: rows of pairs into pages (in eight bits: codes and one exponent per 64 values) and back
    step       rt_decode_step_paged: one position of a layer for sequences at positions of their own, and rt_cache_read of the new pairs
    readout    rt_lm_head_mx4: final norm and output projection with 4-bit weights, one scale per block of 32

Heads are 64 wide.  A sequence of length -1 is an idle place of a padded batch: its rows stay as they were.
"""
import math

import torch

own = False   # True: the library's entry points; False: the plain forms below

DEVICE = "cuda:0"
MATRICES = ("Wq", "Wk", "Wv", "Wo", "W1", "W2")
GAINS = ("g_attn", "g_mlp", "g_kv", "g_q", "g_k")
EPS = 1e-6
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # the first tokens of one conversation: the smallest call, all latency
        dict(name="attention_first_tokens", kind="attention", dtype="bf16", bits=0, S=1, H=8, L=37, page=16, alibi=0.0, scale=1.0, pair=True),
        # an fp32 layer's odd batch, with empty and idle places, without the layer's temporary pair
        dict(name="attention_f32_ragged", kind="attention", dtype="f32", bits=0, S=7, H=2, L=513, page=32, alibi=8.0, scale=0.125, pair=False),
        # conversations of a chat server, cache in eight bits
        dict(name="attention_chat_8bit", kind="attention", dtype="bf16", bits=8, S=64, H=16, L=2000, page=64, alibi=8.0, scale=1.0, pair=True),
        # two long documents: few rows, the work lies along the cache
        dict(name="attention_long", kind="attention", dtype="bf16", bits=0, S=2, H=16, L=100001, page=256, alibi=0.0, scale=0.125, pair=True),
        # a full server: 200 sequences of up to 4096 tokens
        dict(name="attention_full_server", kind="attention", dtype="bf16", bits=0, S=200, H=16, L=4096, page=64, alibi=0.0, scale=1.0, pair=True),
        # one generated token of every sequence of that server, cached and read back
        dict(name="cache_one_token", kind="cache", dtype="bf16", bits=8, S=200, N=1, H=16, page=64),
        # an odd fp32 batch of short prompts
        dict(name="cache_f32_prompts", kind="cache", dtype="f32", bits=8, S=3, N=777, H=2, page=32),
        # eight ragged prompts of up to 2048 tokens (the headline layer) moved into pages
        dict(name="cache_prompts", kind="cache", dtype="bf16", bits=8, S=8, N=2048, H=16, page=64),
        # one token of one conversation through one layer
        dict(name="step_one_sequence", kind="step", dtype="bf16", bits=0, S=1, L=200, d=512, page=16, alibi=0.0, scale=0.125),
        # one token of a serving batch through one layer, cache in eight bits
        dict(name="step_server_8bit", kind="step", dtype="bf16", bits=8, S=200, L=1000, d=1024, page=64, alibi=8.0, scale=0.125),
        # the read-out of one token over the benchmark's vocabulary
        dict(name="readout_one_token", kind="readout", dtype="bf16", B=1, d=1024, vocab=32768),
        # the read-out of a batch over a larger, odd vocabulary
        dict(name="readout_batch", kind="readout", dtype="bf16", B=64, d=1024, vocab=50001),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attention", "attention", "cache", "step", "readout"))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    page, bits = rng.choice((16, 32, 64, 128, 256)), rng.choice((0, 8))
    alibi, scale = rng.choice((0.0, 8.0)), rng.choice((1.0, 0.125))
    if kind == "attention":
        S, H = _log(rng, 1, 256), rng.randint(1, 20)
        rows = 6_500_000 if dtype == "bf16" else 3_000_000   # of 64 values in each of the two pools
        return dict(kind=kind, dtype=dtype, bits=bits, S=S, H=H, L=_log(rng, 1, max(2, min(100_000, rows // (S * H)))), page=page,
                    alibi=alibi, scale=scale, pair=rng.random() < 0.7)
    if kind == "cache":
        S, H = _log(rng, 1, 256), rng.randint(1, 20)
        return dict(kind=kind, dtype=dtype, bits=bits, S=S, N=_log(rng, 1, max(2, min(4096, 400_000 // (S * H)))), H=H, page=page)
    if kind == "step":
        S = _log(rng, 1, 200) if dtype == "bf16" else _log(rng, 1, 12)
        return dict(kind=kind, dtype=dtype, bits=bits, S=S, L=_log(rng, 1, 200_000 // S if S > 40 else 4000),
                    d=rng.choice((256, 320, 512, 1024)) if dtype == "bf16" else rng.choice((128, 256)), page=page, alibi=alibi, scale=0.125)
    return dict(kind=kind, dtype=dtype, B=_log(rng, 1, 64), d=64 * rng.randint(1, 24), vocab=_log(rng, 50, 50000))


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---------------------------------------------------------------------------------------------- inputs
def _normal(g, case, *shape, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=g, device=DEVICE) * std + mean).to(_dtype(case))


def _lengths(g, S, most):
    """Lengths 0 .. most; with four sequences and more one of every border kind: the longest, an empty and an idle place."""
    n = torch.randint(0, most + 1, (S,), generator=g, device=DEVICE, dtype=torch.int32)
    n[0] = most
    if S >= 4:
        n[1], n[2] = 0, -1
    return n


def _pool(g, case, H, pages, filled):
    """K, V [pages, H, page, 64]; keys as the layer's per-head normalisation leaves them, values as its projection does."""
    shape = (pages, H, case["page"], 64)
    if not filled:
        K, V = torch.zeros(shape, device=DEVICE, dtype=_dtype(case)), torch.zeros(shape, device=DEVICE, dtype=_dtype(case))
    else:
        K, V = torch.empty(shape, device=DEVICE, dtype=_dtype(case)), torch.empty(shape, device=DEVICE, dtype=_dtype(case))
        for rows in K.split(max(1, (1 << 25) // (H * case["page"] * 64))):
            u = torch.randn(rows.shape, generator=g, device=DEVICE)
            rows.copy_(u / u.square().mean(-1, keepdim=True).sqrt_())
        for rows in V.split(max(1, (1 << 25) // (H * case["page"] * 64))):
            rows.copy_(torch.randn(rows.shape, generator=g, device=DEVICE) * 0.6)
    if not case["bits"]:
        return dict(K=K, V=V, K_exp=None, V_exp=None)
    (K, ke), (V, ve) = _quantise(K), _quantise(V)
    return dict(K=K, V=V, K_exp=ke, V_exp=ve)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    kind, s = case["kind"], dict(case=case, stream=torch.cuda.current_stream().cuda_stream)
    if kind == "readout":
        d, B = case["d"], case["B"]
        # what is packed ahead: codes of two weights a byte, the even index in the low half, and one exponent byte per block of 32
        w = torch.randn((case["vocab"], d // 32, 32), generator=g, device=DEVICE) * 0.02
        e = torch.frexp(w.abs().amax(-1) / 6.0)[1].clamp_(-126, 127)   # the largest weight of a block is at most 6 steps
        u = torch.ldexp(w, -e[..., None])
        mag = torch.bucketize(u.abs(), torch.tensor((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0), device=DEVICE))
        code = (mag + 8 * (u < 0)).to(torch.uint8).reshape(case["vocab"], d)
        s["codes"], s["exps"] = code[:, 0::2] | (code[:, 1::2] << 4), (e + 127).to(torch.uint8)
        s["g_final"], s["z"] = _normal(g, case, d, std=0.1, mean=1.0), _normal(g, case, B, d)
        s["logits"] = torch.zeros((B, case["vocab"]), device=DEVICE)
        return s
    S, page = case["S"], case["page"]
    H = case["d"] // 64 if kind == "step" else case["H"]
    room = case["N"] + 2 * page if kind == "cache" else case["L"] + 1   # positions that a sequence has pages for
    per = -(-room // page)
    s["table"] = torch.randperm(S * per, generator=g, device=DEVICE).to(torch.int32).reshape(S, per)
    s["pool"] = _pool(g, case, H, S * per, kind != "cache")
    if kind == "cache":
        N = case["N"]
        s["k"], s["v"] = _normal(g, case, N, S, H, 64).transpose(0, 1), _normal(g, case, N, S, H, 64, std=0.6).transpose(0, 1)   # position first
        s["first"] = torch.randint(0, 2 * page, (S,), generator=g, device=DEVICE, dtype=torch.int32)
        s["count"] = _lengths(g, S, N).clamp_(min=0)
        if S >= 4:
            s["first"][2] = -1   # an idle place
        s["k_out"], s["v_out"] = (torch.zeros((S, N, H, 64), device=DEVICE, dtype=_dtype(case)) for _ in range(2))
        return s
    s["lens"] = _lengths(g, S, case["L"])
    if kind == "attention":
        s["q"] = _normal(g, case, S, H, 64)
        s["k_t"], s["v_t"] = (_normal(g, case, S, H, 64), _normal(g, case, S, H, 64, std=0.6)) if case["pair"] else (None, None)
        s["out"] = torch.zeros((S, H, 64), device=DEVICE, dtype=_dtype(case))
        s["lse"] = torch.zeros((S, H), device=DEVICE)
        return s
    d = case["d"]
    w = {n: _normal(g, case, *shape, std=0.02) for n, shape in zip(MATRICES, ((d, d), (d, d), (d, d), (d, d), (4 * d, d), (d, 4 * d)))}
    w.update({n: _normal(g, case, d, std=0.1, mean=1.0) for n in GAINS})
    s["weights"], s["x"] = w, _normal(g, case, S, d)
    s["y"] = torch.zeros((S, d), device=DEVICE, dtype=_dtype(case))
    s["k_out"], s["v_out"] = (torch.zeros((S, 1, H, 64), device=DEVICE, dtype=_dtype(case)) for _ in range(2))
    s["one"] = torch.ones((S,), device=DEVICE, dtype=torch.int32)
    return s


# ---------------------------------------------------------------------------------------------- the library's calls
_contexts, MOST_CONTEXTS = {}, 64


def _context(s, binding):
    """The context that a server keeps for its layers: one per shape and stream, whatever the batch in hand holds.  A state is run on the
    stream that it was prepared on."""
    case = s["case"]
    d, rows = case.get("d") or 64 * case["H"], case.get("S") or case["B"]
    key = (d, rows, case["dtype"], case.get("alibi", 0.0), case.get("scale", 1.0), s["stream"])
    if key not in _contexts:
        if len(_contexts) >= MOST_CONTEXTS:   # the oldest goes, when the device is done with it
            torch.cuda.synchronize()
            _contexts.pop(next(iter(_contexts))).rt_destroy()
        _contexts[key] = binding.RTContext(d, d // 64, 4 * d, rows, 1, case["dtype"], attn_scale=key[4], rms_eps=EPS, alibi_max_bias=key[3],
                                           stream=s["stream"], reserve=binding.RT_RESERVE_PAGED)
    return _contexts[key]


def _run_own(s):
    from paper_2604_21215_amd import binding

    case = s["case"]
    ctx, kind = _context(s, binding), case["kind"]
    if kind == "readout":
        ctx.rt_lm_head_mx4(s["codes"], s["exps"], s["g_final"], s["z"], case["d"], case["B"], s["logits"])
        return s["logits"]
    p = s["pool"]
    cache = binding.make_cache(p["K"], p["V"], s["table"], p["K_exp"], p["V_exp"])
    if kind == "attention":
        ctx.rt_paged_attention(cache, s["lens"], case["L"], s["q"], s["k_t"], s["v_t"], s["out"], s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "cache":
        ctx.rt_cache_write(cache, s["first"], s["count"], s["k"], s["v"])
        ctx.rt_cache_read(cache, s["first"], s["count"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    ctx.rt_decode_step_paged(binding.make_weights(s["weights"]), cache, s["x"], s["lens"], case["L"], s["y"])
    ctx.rt_cache_read(cache, s["lens"], s["one"], s["k_out"], s["v_out"])
    return {"y": s["y"], "k": s["k_out"], "v": s["v_out"]}


# ---------------------------------------------------------------------------------------------- the plain forms
def _quantise(u):
    """Rows of 64 -> int8 codes and exponent bytes: the smallest power of two whose 127 steps hold the row's largest value."""
    f = u.float()
    top = f.abs().amax(-1)
    mant, e = torch.frexp(top)
    e = torch.clamp(e - 7 + (mant > 127 / 128), min=-126)
    fine = torch.isfinite(top)
    e = torch.where(fine, e, 0)
    code = torch.round(torch.ldexp(f, -e[..., None]))
    code = torch.where(fine[..., None], code, 0.0).to(torch.int8)
    byte = torch.where(fine, torch.where(top > 0, e + 127, 0), 255)
    return code, byte.to(torch.uint8)


def _values(codes, exps):
    """What the pool's rows stand for, in 32 bits."""
    if exps is None:
        return codes.float()
    e = exps.int()
    step = torch.ldexp(torch.ones((), device=codes.device), e - 127)
    return codes.float() * torch.where(e == 255, math.nan, torch.where(e == 0, 0.0, step))[..., None]


def _rows_of(pool, exps, table, page, pos):
    """Pool rows of positions pos [S, n]: [S, n, H, 64] in 32 bits."""
    at = torch.gather(table.long(), 1, pos // page), pos % page
    return _values(pool[at[0], :, at[1]], None if exps is None else exps[at[0], :, at[1]])


def _put(pool, exps, table, page, pos, live, u):
    """u [S, n, H, 64] into the rows of positions pos where live."""
    some = live.flatten().to(torch.int32).argmax()   # rows that are not live write one that is once more
    src = torch.where(live.flatten(), torch.arange(live.numel(), device=live.device), some)
    p = torch.where(live, pos, 0)
    page_of = torch.gather(table.long(), 1, p // page).flatten()[src]
    row = (p % page).flatten()[src]
    rows = u.reshape(-1, *u.shape[2:])[src]
    if exps is None:
        pool[page_of, :, row] = rows.to(pool.dtype)
        return
    codes, byte = _quantise(rows)
    pool[page_of, :, row] = codes
    exps[page_of, :, row] = byte


def _attend(s, q, k_t, v_t, H):
    """softmax over the cached rows below lens and the pair at distance 0 -> ([S, H, 64], log-sum-exp [S, H]), 32 bits."""
    case, p, n = s["case"], s["pool"], s["lens"]
    L = case["L"]
    pos = torch.arange(max(L, 1), device=DEVICE).expand(case["S"], -1)
    K = _rows_of(p["K"], p["K_exp"], s["table"], case["page"], pos).transpose(1, 2).contiguous()   # [S, H, L, 64]
    logits = torch.matmul(K, q[..., None]).squeeze(-1) * case["scale"]
    del K
    if case["alibi"]:
        slope = torch.exp2(-case["alibi"] * torch.arange(1, H + 1, device=DEVICE, dtype=torch.float32) / H)
        logits = logits - slope[:, None] * (n[:, None] - pos)[:, None].float()
    logits = torch.where((pos < n[:, None])[:, None], logits, -math.inf)
    if k_t is not None:
        logits = torch.cat((logits, (q * k_t).sum(-1, keepdim=True) * case["scale"]), -1)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = torch.exp(logits - top)
    total = w.sum(-1, keepdim=True)
    V = _rows_of(p["V"], p["V_exp"], s["table"], case["page"], pos).transpose(1, 2).contiguous()
    V = torch.where((pos < n[:, None])[:, None, :, None], V, 0.0)
    o = torch.matmul(w[..., None, :pos.shape[1]], V).squeeze(-2)
    if k_t is not None:
        o = o + w[..., -1:] * v_t
    return torch.where(total > 0, o / total, 0.0), (top + torch.log(total)).squeeze(-1)


def _rms(u, g):
    return u * torch.rsqrt(u.square().mean(-1, keepdim=True) + EPS) * g


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "readout":
        c = s["codes"].int()
        table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=DEVICE)
        w = table[torch.stack((c & 15, c >> 4), -1).reshape(case["vocab"], case["d"] // 32, 32)]
        w = torch.ldexp(w, (s["exps"].int() - 127)[..., None]).reshape(case["vocab"], case["d"])
        return torch.matmul(_rms(s["z"].float(), s["g_final"].float()), w.t())
    p, table, page = s["pool"], s["table"], case["page"]
    if kind == "cache":
        at = torch.arange(case["N"], device=DEVICE).expand(case["S"], -1)
        live = (at < s["count"][:, None]) & (s["first"][:, None] >= 0)
        pos = torch.where(live, s["first"][:, None] + at, 0)
        out = []
        for rows, name, dst in ((s["k"], "K", s["k_out"]), (s["v"], "V", s["v_out"])):
            _put(p[name], p[name + "_exp"], table, page, pos, live, rows)
            got = _rows_of(p[name], p[name + "_exp"], table, page, pos).to(dst.dtype)
            out.append(torch.where(live[..., None, None], got, dst))
        return {"k": out[0], "v": out[1]}
    live = s["lens"] >= 0
    if kind == "attention":
        pair = (s["k_t"].float(), s["v_t"].float()) if case["pair"] else (None, None)
        o, lse = _attend(s, s["q"].float(), *pair, case["H"])
        return {"out": torch.where(live[:, None, None], o.to(_dtype(case)), s["out"]), "lse": torch.where(live[:, None], lse, s["lse"])}
    S, d = case["S"], case["d"]
    H = d // 64
    w = {n: t.float() for n, t in s["weights"].items()}
    x = s["x"].float()
    head = lambda u, g: _rms(u.view(S, H, 64), g.view(H, 64))  # noqa: E731
    n = _rms(x, w["g_attn"])
    o, _ = _attend(s, head(n @ w["Wq"].t(), w["g_q"]), head(n @ w["Wk"].t(), w["g_k"]), (n @ w["Wv"].t()).view(S, H, 64), H)
    h = x + o.reshape(S, d) @ w["Wo"].t()
    u = _rms(h, w["g_mlp"]) @ w["W1"].t()
    z = h + (0.5 * u * (1 + torch.erf(u / math.sqrt(2.0)))) @ w["W2"].t()
    m = _rms(z, w["g_kv"])
    pos = torch.where(live, s["lens"], 0).long()[:, None]
    out = []
    for rows, name, dst in ((head(m @ w["Wk"].t(), w["g_k"]), "K", s["k_out"]), ((m @ w["Wv"].t()).view(S, H, 64), "V", s["v_out"])):
        _put(p[name], p[name + "_exp"], table, page, pos, live[:, None], rows[:, None])
        got = _rows_of(p[name], p[name + "_exp"], table, page, pos).to(dst.dtype)
        out.append(torch.where(live[:, None, None, None], got, dst))
    return {"y": torch.where(live[:, None], z.to(_dtype(case)), s["y"]), "k": out[0], "v": out[1]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------------------- cost and exact values
def _expected(S, most):
    """The sum of _lengths on average."""
    return most * (1 + (S - (3 if S >= 4 else 1)) / 2)


def work(case):
    kind, E = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind == "readout":
        B, d, vocab = case["B"], case["d"], case["vocab"]
        return {"bytes": vocab * d * (0.5 + 1 / 32) + B * d * E + d * E + 4.0 * B * vocab, "flops": 2.0 * B * d * vocab}
    H = case["d"] // 64 if kind == "step" else case["H"]
    S = case["S"]
    row = H * (65 if case["bits"] else 64 * E)   # one position's keys, or its values
    if kind == "cache":
        rows = _expected(S, case["N"])
        return {"bytes": rows * 2 * (2 * H * 64 * E + 2 * row), "flops": rows * 2 * H * 64 * 2}
    live = _expected(S, case["L"])
    by, fl = live * 2 * row, H * 256.0 * (live + S)
    if kind == "attention":
        return {"bytes": by + S * H * 64 * E * (4 if case["pair"] else 2) + 4.0 * S * H, "flops": fl}
    d = case["d"]
    return {"bytes": by + 12.0 * d * d * E + 2.0 * S * d * E + S * 2.0 * (2 * row + H * 64 * E), "flops": fl + S * 28.0 * d * d}


def _wide(pool, exps, pages, n):
    """The first n positions of the pages listed, from their definition in 64 bits: [H, n, 64]."""
    u = pool[pages].double()
    if exps is not None:
        u = u * (2.0 ** (exps[pages].double() - 127.0)).unsqueeze(-1)
    return u.permute(1, 0, 2, 3).reshape(u.shape[1], -1, 64)[:, :n]


def _exact_attention(s, q, k_t, v_t, out, lse):
    case, p = s["case"], s["pool"]
    H = q.shape[1]
    slopes = torch.tensor([2.0 ** (-case["alibi"] * (h + 1) / H) if case["alibi"] else 0.0 for h in range(H)], dtype=torch.float64, device=DEVICE)
    for i, n in enumerate(s["lens"].tolist()):
        if n < 0:
            continue
        parts, values = [], []
        if n:
            pages = s["table"][i, :-(-n // case["page"])].long()
            back = torch.arange(n, 0, -1, device=DEVICE, dtype=torch.float64)
            parts.append((_wide(p["K"], p["K_exp"], pages, n) * q[i][:, None]).sum(-1) * case["scale"] - slopes[:, None] * back)
            values.append(_wide(p["V"], p["V_exp"], pages, n))
        if k_t is not None:
            parts.append((q[i] * k_t[i]).sum(-1, keepdim=True) * case["scale"])
            values.append(v_t[i][:, None])
        if not parts:
            out[i], lse[i] = 0.0, -math.inf
            continue
        logits = torch.cat(parts, 1)
        lse[i] = torch.logsumexp(logits, 1)
        out[i] = (torch.softmax(logits, 1)[..., None] * torch.cat(values, 1)).sum(1)
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "readout":
        low, high = (s["codes"] & 15).long(), (s["codes"] >> 4).long()
        code = torch.stack((low, high), 2).flatten(1)
        w = torch.tensor(E2M1, dtype=torch.float64, device=DEVICE)[code % 8] * (1.0 - 2.0 * (code >= 8))
        w = w * (2.0 ** (s["exps"].double() - 127)).repeat_interleave(32, 1)
        z = s["z"].double()
        z = z / torch.sqrt((z * z).mean(1, keepdim=True) + EPS) * s["g_final"].double()
        return z @ w.t()
    if kind == "cache":
        out = {}
        for name, rows in (("k", s["k"]), ("v", s["v"])):
            at = torch.arange(case["N"], device=DEVICE)[None]
            live = (at < s["count"][:, None]) & (s["first"][:, None] >= 0)
            u = rows.double()
            if case["bits"]:
                top = u.abs().amax(-1, keepdim=True)
                step = 2.0 ** torch.floor(torch.log2(torch.clamp(top, min=1e-300)) - 7.5)   # at most half of what is needed
                step = step * torch.where(top > 127 * step, 2.0, 1.0)
                step = step * torch.where(top > 127 * step, 2.0, 1.0)
                u = torch.where(top > 0, torch.round(u / step) * step, 0.0)
            out[name] = torch.where(live[..., None, None], u, 0.0)
        return out
    out = torch.zeros((case["S"], s["pool"]["K"].shape[1], 64), dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device=DEVICE)
    if kind == "attention":
        pair = (s["k_t"].double(), s["v_t"].double()) if case["pair"] else (None, None)
        out, lse = _exact_attention(s, s["q"].double(), *pair, out, lse)
        return {"out": out, "lse": lse}
    d, S = case["d"], case["S"]
    w = {n: t.double() for n, t in s["weights"].items()}
    norm = lambda u, g: u / torch.sqrt((u * u).mean(-1, keepdim=True) + EPS) * g  # noqa: E731
    heads = lambda u, g: norm(u.reshape(S, -1, 64), g.reshape(-1, 64))  # noqa: E731
    x = s["x"].double()
    n = norm(x, w["g_attn"])
    pair = heads(n @ w["Wk"].T, w["g_k"]), (n @ w["Wv"].T).reshape(S, -1, 64)
    a, _ = _exact_attention(s, heads(n @ w["Wq"].T, w["g_q"]), *pair, out, lse)
    h = x + a.reshape(S, d) @ w["Wo"].T
    z = h + torch.nn.functional.gelu(norm(h, w["g_mlp"]) @ w["W1"].T) @ w["W2"].T
    m = norm(z, w["g_kv"])
    live = (s["lens"] >= 0).double()
    if case["bits"]:   # which of two codes a value next to their border takes is not for 64 bits to say
        return {"y": z * live[:, None], "k": None, "v": None}
    return {"y": z * live[:, None], "k": (heads(m @ w["Wk"].T, w["g_k"]) * live[:, None, None])[:, None],
            "v": ((m @ w["Wv"].T).reshape(S, 1, -1, 64) * live[:, None, None, None])}
