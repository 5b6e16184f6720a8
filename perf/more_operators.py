"""Attention and rotary positions of a pipeline stage's training step, as measurable cases.

A layer turns its queries and keys by their positions (one axis for text; time, height and width for images and video) and lets every
token attend to those that its mask leaves: earlier ones, of its own document, or of a prefix that all of the document sees.  Scores are capped
by a tanh in some models and get a bias by distance in others.  Steps are forward and backward; a probe of a layer's latency and an answer
given token by token are forward calls of one query over many keys.  `listed` holds such calls; `draw` gives more over the same ranges.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------------ cases
def _rotary(mode, tokens, heads, dim, pairs, axes=1, dtype="bf16", index="int64", pairing="halves", far=0, pad=0):
    """axes: 1 (text), 2 (image), 3 (video); far: position of the first token"""
    return dict(op="rotary", mode=mode, tokens=tokens, heads=heads, dim=dim, pairs=pairs, axes=axes, dtype=dtype, index=index, pairing=pairing,
                far=far, pad=pad)


def _attention(mode, batch, tokens, keys, heads, kv_heads, dim, dtype="bf16", cap=0.0, slopes=False, causal=True, documents=0, padding=0.0,
               prefix=0.0, pad=0):
    """documents: of a sequence (0: no document mask); padding: share of places that belong to none; prefix: share of each document"""
    return dict(op="attention", mode=mode, batch=batch, tokens=tokens, keys=keys, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, cap=cap,
                slopes=slopes, causal=causal, documents=documents, padding=padding, prefix=prefix, pad=pad)


def listed():
    cases = [
        # one new token's queries and keys: latency
        ("rotary_token", _rotary("forward", 1, 40, 128, 64)),
        # a short batch in 32 bits, odd sizes, neighbouring pairs, the last elements of a head not turned
        ("rotary_step_odd", _rotary("step", 777, 5, 82, 37, axes=2, dtype="f32", index="int32", pairing="neighbours", pad=3)),
        # queries and keys (32 + 8 heads) of a sequence whose context began a million tokens before
        ("rotary_step_far", _rotary("step", 4096, 40, 128, 64, dtype="f16", far=1 << 20)),
        # a video's patches, three axes, forward and backward: 335 MB in and as much out of each
        ("rotary_step_video", _rotary("step", 32768, 40, 128, 64, axes=3)),
        # one token of each of 8 answers over long contexts: the keys and values are all there is to read
        ("attention_token", _attention("forward", 8, 1, 32768, 32, 8, 128, causal=False)),
        # one token of each of 64 answers of different lengths, capped scores
        ("attention_tokens_ragged", _attention("forward", 64, 1, 2048, 16, 16, 64, "f16", cap=30.0, causal=False, documents=1, padding=0.5)),
        # a chunk of a long prompt behind what came before it, bias by distance
        ("attention_chunk", _attention("forward", 1, 256, 32768, 32, 8, 128, slopes=True)),
        # a probe of a few tokens, forward and backward: latency
        ("attention_step_probe", _attention("step", 1, 17, 17, 4, 4, 64)),
        # a short batch of odd sizes that is aligned to nothing, with everything that a score can get
        ("attention_step_odd", _attention("step", 2, 515, 515, 6, 2, 72, cap=20.0, slopes=True, documents=3, padding=0.1, prefix=0.2, pad=3)),
        # prompts that are seen as a whole, answers that are not: four sequences of two documents
        ("attention_step_prefix", _attention("step", 4, 1024, 1024, 16, 16, 64, "f16", documents=2, prefix=0.4)),
        # one micro-batch (one sequence packed of documents) of a layer 4,096 wide: what fwd_us and bwd_us stand for
        ("attention_step", _attention("step", 1, 4096, 4096, 32, 8, 128, documents=6, padding=0.03)),
        # the largest: a long sequence, capped scores
        ("attention_step_large", _attention("step", 1, 8192, 8192, 32, 8, 128, cap=50.0)),
    ]
    return [dict(c, name=n) for n, c in cases]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.35:
        while True:
            tokens, heads = _log_int(rng, 1, 65536), _log_int(rng, 1, 64)
            dim = rng.choice([64, 80, 96, 128, 2 * rng.randint(4, 128)])
            if tokens * heads * dim <= 32768 * 40 * 128:
                break
        axes = rng.choice([1, 2, 3])
        pairs = rng.choice([dim // 2, dim // 2, rng.randint(3, dim // 2)])
        return _rotary("forward" if tokens < 16 else rng.choice(["forward", "step"]), tokens, heads, dim, pairs, axes, rng.choice(["bf16", "bf16", "f16", "f32"]),
                       rng.choice(["int32", "int64"]), rng.choice(["halves", "neighbours"]), rng.choice([0, 0, _log_int(rng, 1000, 1 << 21)]),
                       rng.choice([0, 0, 3, 64]))
    kv_heads, group = rng.choice([1, 2, 4, 8, rng.randint(1, 12)]), rng.choice([1, 1, 2, 4, 8, rng.randint(1, 9)])
    heads, dim = kv_heads * group, rng.choice([64, 64, 128, 128, 96, 8 * rng.randint(4, 16), rng.randint(17, 128)])
    kind = rng.choice(["token", "chunk", "step", "step", "step"])
    dtype, cap, slopes, pad = rng.choice(["bf16", "bf16", "f16"]), rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.3, rng.choice([0, 0, 64, 3])
    while True:
        batch = _log_int(rng, 1, 64 if kind == "token" else 8)
        keys = _log_int(rng, 1, 65536 if kind != "step" else 8192)
        tokens = {"token": 1, "chunk": min(keys, _log_int(rng, 2, 1024)), "step": keys}[kind]
        # the largest listed case's products, and its memory in the plain form
        if batch * heads * tokens * keys * max(dim, 64) <= 32 * 8192 * 8192 * 64 and batch * keys * heads * dim <= 8 * 32768 * 32 * 128:
            break
    if kind != "step":
        ragged = kind == "token" and rng.random() < 0.5
        return _attention("forward", batch, tokens, keys, heads, kv_heads, dim, dtype, cap, slopes, causal=kind == "chunk",
                          documents=1 if ragged else 0, padding=round(rng.uniform(0.1, 0.6), 3) if ragged else 0.0, pad=pad)
    documents = rng.choice([0, 0, _log_int(rng, 1, max(1, min(16, keys // 4)))])
    causal = rng.random() < 0.8
    return _attention("step", batch, keys, keys, heads, kv_heads, dim, dtype, cap, slopes, causal, documents,
                      round(rng.uniform(0.01, 0.3), 3) if documents and rng.random() < 0.5 else 0.0,
                      round(rng.uniform(0.05, 0.6), 3) if documents and causal and rng.random() < 0.4 else 0.0, pad)


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _sections(case):
    """pairs of each axis: fewer for time, the same for height and width"""
    n, axes = case["pairs"], case["axes"]
    if axes == 1:
        return [n]
    if axes == 2:
        return [n // 2, n - n // 2]
    return [n // 4, (n - n // 4) // 2, n - n // 4 - (n - n // 4) // 2]


def _rotary_inputs(case, seed):
    g = _generator(seed)
    n, H, d, dt = case["tokens"], case["heads"], case["dim"], DTYPES[case["dtype"]]

    def heads():
        t = torch.empty((n, H * d + case["pad"]), dtype=dt, device="cuda").normal_(0.0, 1.0, generator=g)
        return t[:, :H * d].view(n, H, d)

    i = torch.arange(n, device="cuda")
    if case["axes"] == 1:                                                   # tokens in a row
        pos = (i + case["far"])[None]
    else:                                                                   # frames of side x side patches
        side = max(1, int(round(n ** (1 / case["axes"]))))
        pos = torch.stack([i // (side * side), i // side % side, i % side][-case["axes"]:]) + case["far"]
    s = {"x": heads(), "positions": pos.to(torch.int32 if case["index"] == "int32" else torch.int64)}
    if case["mode"] == "step":
        s["dy"] = heads()
    return s


def _layout(case):
    """(document, in its prefix) of every place of every sequence [batch, keys]: whole numbers and truth values; without documents None"""
    B, K = case["batch"], case["keys"]
    if not case["documents"]:
        return None, None
    rng = np.random.default_rng(K * 1000 + case["documents"])
    ids, pre = np.full((B, K), -1, dtype=np.int32), np.zeros((B, K), dtype=bool)
    for b in range(B):
        # places behind the last document belong to none: as many in every sequence of a step, different ones for answers of different lengths
        share = case["padding"] if case["mode"] == "step" else case["padding"] * 2 * rng.random()
        live = max(min(K, case["documents"]), K - int(round(K * min(share, 0.98))))
        cuts = np.sort(rng.choice(np.arange(1, live), min(live, case["documents"]) - 1, replace=False)) if live > 1 else np.array([], dtype=np.int64)
        for n, (a, e) in enumerate(zip(np.r_[0, cuts], np.r_[cuts, live])):
            ids[b, a:e] = n
            pre[b, a:a + int((e - a) * case["prefix"])] = True
    return ids, pre


def _attention_inputs(case, seed):
    g = _generator(seed)
    B, T, K, H, Hk, d, dt = case["batch"], case["tokens"], case["keys"], case["heads"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]
    pad = case["pad"]

    def block(n, heads, std):
        t = torch.empty((B, n, heads * d + pad), dtype=dt, device="cuda").normal_(0.0, std, generator=g)
        return t[:, :, :heads * d].unflatten(2, (heads, d))

    s = {}
    if case["mode"] == "step":                                              # one projection's result: queries, keys and values side by side
        both = block(T, H + 2 * Hk, 1.2)
        s["q"], s["k"], s["v"] = both[:, :, :H], both[:, :, H:H + Hk], both[:, :, H + Hk:]
        s["dy"] = block(T, H, 0.05)
    else:
        s["q"], s["k"], s["v"] = block(T, H, 1.2), block(K, Hk, 1.2), block(K, Hk, 1.0)
    ids, pre = _layout(case)
    if ids is not None:
        s["k_documents"] = torch.from_numpy(ids).cuda()
        s["q_documents"] = s["k_documents"] if T == K else torch.zeros((B, T), dtype=torch.int32, device="cuda")
        if case["prefix"]:
            s["prefix"] = torch.from_numpy(pre).cuda()
    if case["slopes"]:
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda") / H).float()
    return s


def _inputs(case, seed):
    return (_rotary_inputs if case["op"] == "rotary" else _attention_inputs)(case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own and case["op"] == "rotary":                                      # the description of the positions, made once for a model
        from paper_2508_21613_amd import operators as ops
        s["rotary"] = ops.Rotary(case["dim"], _sections(case), base=10000.0, pairing=case["pairing"])
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _turn(case, x, pos, sign):
    """x turned by sign times its angles"""
    P, dev = case["pairs"], x.device
    axis = torch.repeat_interleave(torch.arange(case["axes"], device=dev), torch.tensor(_sections(case), device=dev), output_size=P)
    freq = torch.pow(10000.0, torch.arange(P, dtype=torch.float64, device=dev) / -P)
    angle = pos.double()[axis].t() * freq                                   # [tokens, pairs]; far positions need 64 bits
    c, s = torch.cos(angle).float()[:, None], sign * torch.sin(angle).float()[:, None]
    f = x.float()
    out = f.clone()
    if case["pairing"] == "halves":
        a, b = f[..., :P], f[..., P:2 * P]
        out[..., :P], out[..., P:2 * P] = a * c - b * s, a * s + b * c
    else:
        a, b = f[..., 0:2 * P:2], f[..., 1:2 * P:2]
        out[..., 0:2 * P:2], out[..., 1:2 * P:2] = a * c - b * s, a * s + b * c
    return out.to(x.dtype)


def _plain_rotary(s):
    case = s["case"]
    out = {"y": _turn(case, s["x"], s["positions"], 1.0)}
    if case["mode"] == "step":
        out["dx"] = _turn(case, s["dy"], s["positions"], -1.0)
    return out


def _own_rotary(s):
    out = {"y": s["rotary"].rotate(s["x"], s["positions"])}
    if s["case"]["mode"] == "step":
        out["dx"] = s["rotary"].gradient(s["dy"], s["positions"])
    return out


def _visible(s):
    """[batch or 1, tokens, keys], None: all"""
    case = s["case"]
    T, K, dev = case["tokens"], case["keys"], s["q"].device
    m = None
    if case["causal"]:
        m = (torch.arange(K, device=dev)[None, :] <= torch.arange(T, device=dev)[:, None] + (K - T))[None]
        if "prefix" in s:
            m = m | s["prefix"][:, None, :]
    if "k_documents" in s:
        same = (s["q_documents"][:, :, None] == s["k_documents"][:, None, :]) & (s["k_documents"] >= 0)[:, None, :]
        m = same if m is None else m & same
    return m


def _plain_attention(s):
    case = s["case"]
    B, T, K, H, Hk, d, dt = case["batch"], case["tokens"], case["keys"], case["heads"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]
    G, scale, cap = H // Hk, d ** -0.5, case["cap"]

    def by_head(t, g):                                                      # [batch, kv head, group x tokens, dim]
        return t.float().unflatten(2, (Hk, g)).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, d)

    def back(t, g, n):
        return t.unflatten(2, (g, n)).permute(0, 3, 1, 2, 4).reshape(B, n, Hk * g, d).to(dt)

    q, k, v = by_head(s["q"], G), by_head(s["k"], 1), by_head(s["v"], 1)
    p = torch.matmul(q, k.transpose(2, 3)).mul_(scale)
    t = None
    if cap:
        t = p.div_(cap).tanh_()
        p = t * cap
    p = p.view(B, Hk, G, T, K)
    if "slopes" in s:
        far = (torch.arange(T, device=p.device)[:, None] + (K - T) - torch.arange(K, device=p.device)).abs().float()
        p.sub_(s["slopes"].view(Hk, G, 1, 1) * far)
    seen = _visible(s)
    if seen is not None:
        p.masked_fill_(~seen[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total == 0, 1.0, total))                             # a row that sees nothing: zeros
    p = p.view(B, Hk, G * T, K)
    out = {"y": back(torch.matmul(p, v), G, T)}
    if case["mode"] == "forward":
        return out
    dy = by_head(s["dy"], G)
    out["dv"] = back(torch.matmul(p.transpose(2, 3), dy), 1, K)
    ds = torch.matmul(dy, v.transpose(2, 3))
    ds.sub_((ds * p).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    if cap:
        ds.mul_(1 - t * t)
    out["dq"] = back(torch.matmul(ds, k), G, T)
    out["dk"] = back(torch.matmul(ds.transpose(2, 3), q), 1, K)
    return out


def _own_attention(s):
    from paper_2508_21613_amd import operators as ops
    case = s["case"]
    kw = dict(cap=case["cap"], causal=case["causal"], slopes=s.get("slopes"), prefix=s.get("prefix"))
    if "k_documents" in s:
        kw["documents"] = s["k_documents"] if case["tokens"] == case["keys"] else (s["q_documents"], s["k_documents"])
    if case["mode"] == "forward":
        return {"y": ops.attention_forward(s["q"], s["k"], s["v"], **kw)}
    y, saved = ops.attention_forward(s["q"], s["k"], s["v"], save=True, **kw)
    dq, dk, dv = ops.attention_backward(s["dy"], s["q"], s["k"], s["v"], y, saved, **kw)
    return {"y": y, "dq": dq, "dk": dk, "dv": dv}


def run(state):
    op = state["case"]["op"]
    if own:
        return (_own_rotary if op == "rotary" else _own_attention)(state)
    return (_plain_rotary if op == "rotary" else _plain_attention)(state)


# ------------------------------------------------------------------------------------------------ floors
def _pairs(case):
    """visible pairs of a query and a key, over the batch, for one head"""
    B, T, K = case["batch"], case["tokens"], case["keys"]
    ids, pre = _layout(case)
    if ids is None:
        return B * (T * (2 * K - T + 1) // 2 if case["causal"] else T * K)
    if T != K:
        return int((ids >= 0).sum()) * T
    n = 0
    for b in range(B):
        for doc in range(ids[b].max() + 1):
            here = ids[b] == doc
            size, before = int(here.sum()), int((here & pre[b]).sum())
            n += size * (size + 1) // 2 + before * (before - 1) // 2 if case["causal"] else size * size
    return n


def work(case):
    e, d = SIZE[case["dtype"]], case["dim"]
    if case["op"] == "rotary":
        n, passes = case["tokens"] * case["heads"], 2 if case["mode"] == "step" else 1
        return {"bytes": passes * 2 * n * d * e + case["axes"] * case["tokens"] * (4 if case["index"] == "int32" else 8), "flops": passes * 6 * n * case["pairs"]}
    B, T, K, H, Hk = case["batch"], case["tokens"], case["keys"], case["heads"], case["kv_heads"]
    queries, keys = B * T * H * d * e, B * K * Hk * d * e
    ids, _ = _layout(case)
    if ids is not None and T != K:
        keys = int((ids >= 0).sum()) * Hk * d * e                           # the places of no document are not needed
    step = case["mode"] == "step"
    return {"bytes": (4 if step else 2) * queries + (4 if step else 2) * keys, "flops": (14 if step else 4) * d * H * _pairs(case)}


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_rotary(case, s) if case["op"] == "rotary" else _exact_attention(case, s)


def _exact_rotary(case, s):
    P, at, rows = case["pairs"], 0, []
    for axis, n in enumerate(_sections(case)):
        rows += [(axis, 10000.0 ** (-(at + i) / P)) for i in range(n)]
        at += n
    angle = torch.stack([s["positions"][axis].double() * f for axis, f in rows], dim=1)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]           # e^(i theta)

    def turned(x, by):
        x = x.double()
        if case["pairing"] == "halves":
            z = torch.complex(x[..., :P].contiguous(), x[..., P:2 * P].contiguous()) * by
            return torch.cat([z.real, z.imag, x[..., 2 * P:]], dim=-1)
        z = torch.complex(x[..., 0:2 * P:2].contiguous(), x[..., 1:2 * P:2].contiguous()) * by
        return torch.cat([torch.view_as_real(z).flatten(-2), x[..., 2 * P:]], dim=-1)

    out = {"y": turned(s["x"], turn)}
    if case["mode"] == "step":
        out["dx"] = turned(s["dy"], turn.conj())
    return out


def _exact_attention(case, s):
    """one head of one sequence after the other; gradients by autograd"""
    B, T, K, H, Hk, d = (case[k] for k in ("batch", "tokens", "keys", "heads", "kv_heads", "dim"))
    dev, step = s["q"].device, case["mode"] == "step"
    i, j = torch.arange(T, device=dev).unsqueeze(1) + K - T, torch.arange(K, device=dev).unsqueeze(0)
    y = torch.zeros((B, T, H, d), dtype=torch.float64, device=dev)
    grads = [torch.zeros((B, n, h, d), dtype=torch.float64, device=dev) for n, h in ((T, H), (K, Hk), (K, Hk))] if step else []
    for b in range(B):
        hidden = torch.zeros((T, K), dtype=torch.bool, device=dev)
        if case["causal"]:
            hidden |= j > i
            if "prefix" in s:
                hidden &= ~s["prefix"][b]
        if "k_documents" in s:
            dq, dk = s["q_documents"][b].unsqueeze(1), s["k_documents"][b].unsqueeze(0)
            hidden |= (dq != dk) | (dk < 0)
        some = (~hidden).any(1, keepdim=True)                               # rows that see anything
        for h in range(H):
            q, k, v = (t.double().requires_grad_(step) for t in (s["q"][b, :, h], s["k"][b, :, h * Hk // H], s["v"][b, :, h * Hk // H]))
            with torch.set_grad_enabled(step):
                z = torch.mm(q, k.t()) / math.sqrt(d)
                if case["cap"]:
                    z = torch.tanh(z / case["cap"]) * case["cap"]
                if "slopes" in s:
                    z = z - float(s["slopes"][h]) * (i - j).abs()
                z = z.masked_fill(hidden & some, -math.inf)
                o = torch.mm(torch.exp(z - torch.logsumexp(z, 1, keepdim=True)), v) * some
            y[b, :, h] = o.detach()
            if step:
                for total, part, at in zip(grads, torch.autograd.grad(o, (q, k, v), s["dy"][b, :, h].double()), (h, h * Hk // H, h * Hk // H)):
                    total[b, :, at] += part
    return dict(zip(("y", "dq", "dk", "dv"), [y] + grads))
