"""The operators of a pipeline stage's training step, as measurable cases.

The per-layer times that a scenario is made of are those of a training step: the first stage looks tokens up in its embedding,
every layer runs a gated feed-forward block forward and backward, the first stage gathers the embedding's gradient, and the step
ends with the global gradient norm and the clipping.  A step serves lengths from one token (a probe of a layer's latency, an
answer given token by token) to a whole micro-batch.  `listed` holds such calls; `draw` gives more over the same ranges.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------------ cases
def _ffn(mode, T, D, F, dtype="bf16", act="silu", pad=0):
    return dict(op="ffn", mode=mode, T=T, D=D, F=F, dtype=dtype, act=act, pad=pad)


def _embed(mode, n, V, D, dtype="bf16", index="int64", scaled=False, padding=0.0):
    return dict(op="embed", mode=mode, n=n, V=V, D=D, dtype=dtype, index=index, scaled=scaled, padding=padding)


def _clip(kind, size, dtype="bf16", layers=1, clips=True):
    return dict(op="clip", kind=kind, size=size, dtype=dtype, layers=layers, clips=clips)


def listed():
    cases = [
        # one token through a 4096-wide layer: the weights are all there is to read
        ("ffn_token", _ffn("forward", 1, 4096, 11008)),
        # a few sequences answered token by token, an odd number of them, half precision
        ("ffn_tokens", _ffn("forward", 37, 2048, 5504, "f16", "gelu_tanh")),
        # a short ragged micro-batch of a small layer of odd widths: nothing is aligned
        ("ffn_step_odd", _ffn("step", 515, 1000, 2731, act="gelu", pad=3)),
        # one micro-batch (one sequence) of a 4096-wide layer, forward and backward: what fwd_us and bwd_us stand for
        ("ffn_step", _ffn("step", 4096, 4096, 11008)),
        # the largest: two sequences through an 8192-wide layer
        ("ffn_step_large", _ffn("step", 8192, 8192, 22016)),
        # the tokens of a few answers looked up: latency
        ("embed_tokens", _embed("lookup", 5, 32000, 4096)),
        # a small vocabulary with odd rows in 32 bits, gradient of a short micro-batch
        ("embed_step_odd", _embed("step", 300, 1000, 515, "f32", "int32", scaled=True)),
        # the first stage's share of a step: four sequences, lookup and gradient, a few places padded
        ("embed_step", _embed("step", 16384, 32000, 4096, scaled=True, padding=0.06)),
        # many tokens over a large vocabulary
        ("embed_step_large", _embed("step", 65536, 128000, 2048, "f16", "int32")),
        # a handful of small tensors (norms' and biases' gradients): latency
        ("clip_small", _clip("small", 12, "f32")),
        # hundreds of tensors of odd sizes and mixed types, starting anywhere
        ("clip_ragged", _clip("ragged", 300, "mixed")),
        # the gradients of a stage of four layers, 4096 wide
        ("clip_stage", _clip("stage", 4096, "bf16", layers=4)),
    ]
    return [dict(c, name=n) for n, c in cases]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    w, step = 3072, 1
    while w == 3072:
        step = rng.choice([1, 8, 64])
        w = max(step, _log_int(rng, lo, hi) // step * step)
    return w


def draw(rng):
    op = rng.choice(["ffn", "ffn", "embed", "clip"])
    if op == "ffn":
        while True:
            D = _width(rng, 64, 8192)
            F = _width(rng, 2 * D, 4 * D)
            T = _log_int(rng, 1, 8192)
            if T * D * F <= 8192 * 8192 * 22016:
                break
        mode = "forward" if T < 16 else rng.choice(["forward", "step"])
        return _ffn(mode, T, D, F, rng.choice(["bf16", "bf16", "f16"]), rng.choice(["silu", "silu", "gelu", "gelu_tanh"]),
                    rng.choice([0, 0, 64, 3]))
    if op == "embed":
        while True:
            n, V, D = _log_int(rng, 1, 65536), _log_int(rng, 100, 128000), _width(rng, 64, 8192)
            if (n + V) * D <= (65536 + 128000) * 2048:
                break
        return _embed(rng.choice(["lookup", "step", "step"]), n, V, D, rng.choice(["bf16", "f16", "f32"]), rng.choice(["int32", "int64"]),
                      rng.random() < 0.5, rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.5), 3)]))
    kind = rng.choice(["small", "ragged", "stage"])
    size = {"small": _log_int(rng, 1, 40), "ragged": _log_int(rng, 2, 400), "stage": _width(rng, 256, 4096)}[kind]
    return _clip(kind, size, "mixed" if kind == "ragged" else rng.choice(["bf16", "f16", "f32"]),
                 rng.randint(1, 2) if kind == "stage" else 1, rng.random() < 0.75)


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, rows, cols, dtype, std, pad=0):
    """rows x cols normal numbers; `pad` more columns in memory between the rows"""
    t = torch.empty((rows, cols + pad), dtype=dtype, device="cuda")
    t.normal_(0.0, std, generator=g)
    return t[:, :cols]


def _ffn_inputs(case, seed):
    g = _generator(seed)
    T, D, F, dt = case["T"], case["D"], case["F"], DTYPES[case["dtype"]]
    s = {"x": _normal(g, T, D, dt, 1.0, case["pad"]),                       # what a norm hands over
         "w_gate": _normal(g, F, D, dt, D ** -0.5), "w_up": _normal(g, F, D, dt, D ** -0.5),
         "w_down": _normal(g, D, F, dt, F ** -0.5)}
    if case["mode"] == "step":
        s["dy"] = _normal(g, T, D, dt, 0.05, case["pad"])
    return s


def _token_share(V):
    """probability of the r-th most frequent token: falls about as 1/r, as in text"""
    r = np.arange(V, dtype=np.float64)
    return np.log((r + 2) / (r + 1)) / math.log(V + 1)


def _embed_inputs(case, seed):
    g = _generator(seed)
    n, V, D, dt = case["n"], case["V"], case["D"], DTYPES[case["dtype"]]
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1)) - 1).floor().clamp_(0, V - 1).to(torch.int64)
    order = torch.randperm(V, generator=g, device="cuda")                   # frequent tokens lie anywhere in the table
    tokens = order[rank]
    k = int(round(n * case["padding"]))
    if k:
        tokens[n - k:] = -1                                                 # padded places: no token
    s = {"tokens": tokens.to(torch.int32 if case["index"] == "int32" else torch.int64),
         "table": _normal(g, V, D, dt, 0.02)}
    if case["mode"] == "step":
        s["dy"] = _normal(g, n, D, dt, 0.01)
    return s


def _clip_sizes(case):
    """(elements, dtype, offset in elements of the tensor in its buffer) of every tensor"""
    rng = np.random.default_rng(case["size"] * 1000 + case["layers"])
    if case["kind"] == "small":
        return [(int(n), case["dtype"], 0) for n in rng.integers(1, 8192, case["size"])]
    if case["kind"] == "ragged":
        n = np.exp(rng.uniform(0, math.log(1 << 21), case["size"])).astype(np.int64)
        kinds = rng.choice(["bf16", "f16", "f32"], case["size"])
        return [(int(a), str(k), int(o)) for a, k, o in zip(n, kinds, rng.integers(0, 9, case["size"]))]
    W = case["size"]
    H = W * 43 // 16                                                        # 11008 at 4096
    layer = [W * W] * 4 + [W * H] * 3 + [W, W]
    return [(n, case["dtype"], 0) for n in layer * case["layers"]]


def _clip_inputs(case, seed):
    g = _generator(seed)
    grads, expected = [], 0.0
    for i, (n, dt, off) in enumerate(_clip_sizes(case)):
        buf = torch.empty(n + off, dtype=DTYPES[dt], device="cuda")
        buf.normal_(0.0, 0.02 * (1 + i % 5), generator=g)
        grads.append(buf[off:])
        expected += n * (0.02 * (1 + i % 5)) ** 2
    return {"grads": grads, "max_norm": math.sqrt(expected) * (0.3 if case["clips"] else 16.0)}


def _inputs(case, seed):
    return {"ffn": _ffn_inputs, "embed": _embed_inputs, "clip": _clip_inputs}[case["op"]](case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "clip":                                                # the optimizer's copy: one buffer for each type
        s["flat"], s["out"] = _flat(s["grads"])
        if own:
            from paper_2508_21613_amd import operators as ops
            s["list"] = ops.Gradients(s["grads"], s["out"])                 # the buffers stay where they are from step to step
    return s


def _flat(grads):
    """a buffer for each type that the gradients are of, and a place for each of them, one behind the other"""
    flat, places, at = {}, [], {}
    for dt in DTYPES.values():
        n = sum(g.numel() for g in grads if g.dtype == dt)
        if n:
            flat[dt], at[dt] = torch.empty(n, dtype=dt, device="cuda"), 0
    for g in grads:
        places.append(flat[g.dtype][at[g.dtype]:at[g.dtype] + g.numel()])
        at[g.dtype] += g.numel()
    return list(flat.values()), places


def _scale(case):
    return math.sqrt(case["D"]) if case["scaled"] else 1.0


# ------------------------------------------------------------------------------------------------ one pass
def _activation(act, g):
    """the activation of g and its derivative"""
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _plain_ffn(s):
    case = s["case"]
    dt = DTYPES[case["dtype"]]
    x, wg, wu, wd = (s[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    g, u = x @ wg.t(), x @ wu.t()
    a, da = _activation(case["act"], g)
    h = a * u
    y = (h @ wd.t()).to(dt)
    if case["mode"] == "forward":
        return {"y": y}
    dy = s["dy"].float()
    dh = dy @ wd
    du, dg = dh * a, dh * u * da
    return {"y": y, "dx": (dg @ wg + du @ wu).to(dt), "dw_gate": (dg.t() @ x).to(dt), "dw_up": (du.t() @ x).to(dt),
            "dw_down": (dy.t() @ h).to(dt)}


def _own_ffn(s):
    from paper_2508_21613_amd import operators as ops
    case = s["case"]
    w = (s["w_gate"], s["w_up"], s["w_down"])
    if case["mode"] == "forward":
        return {"y": ops.ffn_forward(s["x"], *w, activation=case["act"])}
    y, saved = ops.ffn_forward(s["x"], *w, activation=case["act"], save=True)
    dx, dwg, dwu, dwd = ops.ffn_backward(s["dy"], s["x"], *w, saved, activation=case["act"])
    return {"y": y, "dx": dx, "dw_gate": dwg, "dw_up": dwu, "dw_down": dwd}


def _plain_embed(s):
    case = s["case"]
    dt, V, D = DTYPES[case["dtype"]], case["V"], case["D"]
    tok = s["tokens"].long()
    there = (tok >= 0) & (tok < V)
    row = torch.where(there, tok, 0)
    e = torch.where(there[:, None], s["table"][row].float() * _scale(case), 0.0).to(dt)
    if case["mode"] == "lookup":
        return {"rows": e}
    dw = torch.zeros((V + 1, D), dtype=torch.float32, device="cuda")
    dw.index_add_(0, torch.where(there, tok, V), s["dy"].float() * _scale(case))
    return {"rows": e, "dtable": dw[:V].to(dt)}


def _own_embed(s):
    from paper_2508_21613_amd import operators as ops
    case = s["case"]
    out = {"rows": ops.embedding_lookup(s["tokens"], s["table"], scale=_scale(case))}
    if case["mode"] == "step":
        out["dtable"] = ops.embedding_gradient(s["dy"], s["tokens"], case["V"], scale=_scale(case))
    return out


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    c = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * c)
    return {"norm": norm, "grads": s["flat"]}


def _own_clip(s):
    return {"norm": s["list"].clip(s["max_norm"]), "grads": s["flat"]}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"ffn": _own_ffn, "embed": _own_embed, "clip": _own_clip}[op](state)
    return {"ffn": _plain_ffn, "embed": _plain_embed, "clip": _plain_clip}[op](state)


# ------------------------------------------------------------------------------------------------ floors
def work(case):
    if case["op"] == "ffn":
        T, D, F, e = case["T"], case["D"], case["F"], SIZE[case["dtype"]]
        if case["mode"] == "forward":
            return {"bytes": e * (3 * D * F + 2 * T * D), "flops": 6 * T * D * F}
        return {"bytes": e * (6 * D * F + 4 * T * D), "flops": 18 * T * D * F}
    if case["op"] == "embed":
        n, V, D, e = case["n"], case["V"], case["D"], SIZE[case["dtype"]]
        live = n - int(round(n * case["padding"]))
        used = float(np.sum(1 - (1 - _token_share(V)) ** live))             # different tokens among them
        b = used * D * e + n * D * e + n * (4 if case["index"] == "int32" else 8)
        f = n * D
        if case["mode"] == "step":
            b += live * D * e + V * D * e
            f += 2 * n * D
        return {"bytes": int(b), "flops": f}
    sizes = _clip_sizes(case)
    return {"bytes": sum(2 * n * SIZE[dt] for n, dt, _ in sizes) + 4, "flops": sum(3 * n for n, _, _ in sizes)}


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "ffn":
        return _exact_ffn(case, s)
    if case["op"] == "embed":
        return _exact_embed(case, s)
    total = sum(float(torch.dot(g.double(), g.double())) for g in s["grads"])
    norm = math.sqrt(total)
    c = min(1.0, s["max_norm"] / (norm + 1e-6))
    grads = [torch.cat([g.double() * c for g in s["grads"] if g.dtype == dt])
             for dt in DTYPES.values() if any(g.dtype == dt for g in s["grads"])]
    return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"), "grads": grads}


def _exact_ffn(case, s):
    mm = torch.mm
    X, Wg, Wu, Wd = (s[k].double() for k in ("x", "w_gate", "w_up", "w_down"))
    G = mm(X, Wg.T)
    U = mm(X, Wu.T)
    G.requires_grad_(True)
    if case["act"] == "silu":
        A = G * torch.sigmoid(G)
    elif case["act"] == "gelu":
        A = G * torch.special.ndtr(G)
    else:
        A = G * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (G + 0.044715 * G ** 3))
    dA = torch.autograd.grad(A.sum(), G)[0] if case["mode"] == "step" else None
    A = A.detach()
    H = A * U
    out = {"y": mm(H, Wd.T)}
    if case["mode"] == "forward":
        return out
    dY = s["dy"].double()
    out["dw_down"] = mm(dY.T, H)
    dH = mm(dY, Wd)
    dG, dU = dH * U * dA, dH * A
    del dH, H, A, dA, U, G
    out["dx"] = mm(dG, Wg).add_(mm(dU, Wu))
    out["dw_gate"] = mm(dG.T, X)
    out["dw_up"] = mm(dU.T, X)
    return {k: out[k] for k in ("y", "dx", "dw_gate", "dw_up", "dw_down")}


def _exact_embed(case, s):
    V, scale = case["V"], _scale(case)
    tok = s["tokens"].long()
    live = torch.nonzero((tok >= 0) & (tok < V)).flatten()
    rows = torch.zeros((case["n"], case["D"]), dtype=torch.float64, device="cuda")
    rows[live] = s["table"][tok[live]].double() * scale
    if case["mode"] == "lookup":
        return {"rows": rows}
    order = live[torch.argsort(tok[live], stable=True)]                     # sums over runs of equal tokens
    dw = torch.zeros((V, case["D"]), dtype=torch.float64, device="cuda")
    which, counts = torch.unique_consecutive(tok[order], return_counts=True)
    if len(order):
        for c in range(0, case["D"], 512):
            part = torch.segment_reduce(s["dy"][order, c:c + 512].double(), "sum", lengths=counts, axis=0)
            dw[which, c:c + 512] = part * scale
    return {"rows": rows, "dtable": dw}
