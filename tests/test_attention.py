"""Attention on the GPU against its formulas in 64 bits.

Tolerances.  Weights p and their gradients ds enter products rounded to the tensors' type of unit roundoff u: each is off by at most u of itself
(in float16 at least 2^-25), independently, with a standard deviation of that bound / sqrt(3).  dy.y is taken with y as it was stored, rounded
once: that error is common to a row of ds.  Scores are float32 sums of dim products, and the exponential's argument is rounded a few times: 2^-24 of
its terms.  The sum of these variances is worked out for every element of the results; an error of six standard deviations and the rounding of the
result itself is allowed.  A pair that is seen or left out wrongly, or a sum that misses a tile, is tens of times that.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
ACC = 2.0 ** -24
BOTH = [torch.bfloat16, torch.float16]
NAMES = ("dq", "dk", "dv")


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_21613_amd import binding, operators
    binding.lib()
    return operators


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, shape, dtype, std=1.0, pad=0, shift=0):
    """[batch, tokens, heads, dim] of normal numbers; tokens `pad` elements further apart than they are long, the first `shift` into its buffer"""
    B, T, H, d = shape
    buf = torch.full((B * T * (H * d + pad) + shift,), float("nan"), dtype=dtype, device="cuda")
    t = buf[shift:].view(B, T, H * d + pad)[:, :, :H * d].unflatten(2, (H, d))
    t.copy_(torch.randn(shape, generator=g, device="cuda") * std)
    return t


def inputs(seed, B, T, K, H, Hk, d, dtype, pad=0, shift=0):
    g = gen(seed)
    return [normal(g, s, dtype, std, pad, shift) for s, std in (((B, T, H, d), 1.5), ((B, K, Hk, d), 1.5), ((B, K, Hk, d), 1.0), ((B, T, H, d), 0.3))]


def visible(B, T, K, causal=True, documents=None, prefix=None):
    i, j = torch.arange(T, device="cuda")[:, None] + K - T, torch.arange(K, device="cuda")[None]
    see = torch.ones((B, T, K), dtype=torch.bool, device="cuda")
    if causal:
        see &= j <= i
        if prefix is not None:
            see |= prefix.bool()[:, None, :]
    if documents is not None:
        dq, dk = documents if isinstance(documents, tuple) else (documents, documents)
        see &= (dq[:, :, None] == dk[:, None, :]) & (dk >= 0)[:, None, :] & (dk < 2 ** 31 - 1)[:, None, :]
    return see


def clean(t, documents, which):
    """zeros in the places of no document: what lies there is no input"""
    t = t.double()
    if documents is None:
        return t
    ids = documents[which] if isinstance(documents, tuple) else documents
    return torch.where(((ids >= 0) & (ids < 2 ** 31 - 1))[:, :, None, None], t, 0.0)


def formula(q, k, v, dy=None, scale=None, cap=0.0, slopes=None, causal=True, documents=None, prefix=None, kept=1.0):
    """{name: (value, variance of the error)} in 64 bits, one key head after the other.  kept: share of their roundings that p and ds have in the gradients'
    products"""
    dtype, (B, T, H, d), (K, Hk) = q.dtype, q.shape, k.shape[1:3]
    u, tiny, G = U[dtype], TINY[dtype], H // Hk
    scale = d ** -0.5 if scale is None else scale
    see = visible(B, T, K, causal, documents, prefix)
    far = (torch.arange(T, device="cuda")[:, None] + K - T - torch.arange(K, device="cuda")[None]).abs().double()
    q, k, v = clean(q, documents, 0), clean(k, documents, 1), clean(v, documents, 1)
    dy = None if dy is None else clean(dy, documents, 0)
    out = {n: (torch.zeros(s, dtype=torch.float64, device="cuda"), torch.zeros(s, dtype=torch.float64, device="cuda"))
           for n, s in (("y", q.shape), ("dq", q.shape), ("dk", k.shape), ("dv", v.shape))}

    def put(name, b, at, value, var):
        out[name][0][b, :, at] += value
        out[name][1][b, :, at] += var

    for b in range(B):
        for h in range(H):
            qq, kk, vv = q[b, :, h], k[b, :, h // G], v[b, :, h // G]
            x = scale * qq @ kk.T
            e = scale * ACC * math.sqrt(d) * ((qq * qq) @ (kk * kk).T).sqrt() + 2 * ACC * x.abs()
            dz = torch.ones_like(x)
            z, more = x, torch.zeros_like(x)
            if cap:
                t = torch.tanh(x / cap)
                z, dz = cap * t, 1 - t * t
                more = 8 * ACC + 2 * e / cap                     # of dz
                e = e * dz + (4 * ACC * cap if cap <= 256 else 16 * ACC * z.abs())       # of a series or the tanh from 1 / 4 on
            s = z - (float(slopes[h]) * far if slopes is not None else 0.0)
            s = s.masked_fill(~see[b], -math.inf)
            some = see[b].any(1, keepdim=True)
            lse = torch.where(some, torch.logsumexp(s, 1, keepdim=True), 0.0)
            p = torch.exp(s - lse)
            e = e + ACC * (4 * torch.where(see[b], s, 0.0).abs() + 4 * lse.abs() + 8)
            vp = ((u * p) ** 2 + torch.where(see[b], tiny, 0.0) ** 2) / 3
            y = p @ vv
            pe = (p * e) ** 2
            vy = vp @ (vv * vv) + 2 * (pe @ (vv * vv) + y * y * pe.sum(1, keepdim=True)) + ACC ** 2 * K * ((p * p) @ (vv * vv)) + (8 * ACC * y) ** 2
            put("y", b, h, y, vy)
            if dy is None:
                continue
            gy = dy[b, :, h]
            dp = gy @ vv.T
            vdp = ACC ** 2 * d * ((gy * gy) @ (vv * vv).T)
            delta = (gy * y).sum(1, keepdim=True)
            vdelta = ((gy * gy) * (vy + (u * y).clamp(min=tiny) ** 2 / 3)).sum(1, keepdim=True) + ACC ** 2 * d * ((gy * y) ** 2).sum(1, keepdim=True)
            ds = p * (dp - delta) * dz
            vds = (p * dz) ** 2 * vdp + (ds * e) ** 2 + (p * (dp - delta) * more) ** 2 + (8 * ACC * p * dp * dz) ** 2 + (
                (kept * u * ds) ** 2 + torch.where(see[b], tiny, 0.0) ** 2) / 3
            pz = p * dz
            vp = ((kept * u * p) ** 2 + torch.where(see[b], tiny, 0.0) ** 2) / 3
            dq, dk, dv = scale * ds @ kk, scale * ds.T @ qq, p.T @ gy
            put("dq", b, h, dq, scale ** 2 * (vds @ (kk * kk) + vdelta * (pz @ kk) ** 2 + ACC ** 2 * K * ((ds * ds) @ (kk * kk))) + (8 * ACC * dq) ** 2)
            put("dk", b, h // G, dk, scale ** 2 * ((vds + pz * pz * vdelta).T @ (qq * qq) + ACC ** 2 * T * G * ((ds * ds).T @ (qq * qq))) + (8 * ACC * dk) ** 2)
            put("dv", b, h // G, dv, (vp + pe).T @ (gy * gy) + ACC ** 2 * T * G * ((p * p).T @ (gy * gy)) + (8 * ACC * dv) ** 2)
    return out if dy is not None else {"y": out["y"]}


def check(name, got, want):
    value, var = want
    assert got.shape == value.shape, name
    assert bool(torch.isfinite(got).all()), name
    err = (got.double() - value).abs()
    tol = 6 * var.sqrt() + torch.clamp(value.abs() * U[got.dtype], min=TINY[got.dtype]) * 1.0001 + 1e-30
    bad = err > tol
    assert not bool(bad.any()), (name, int(bad.sum()), float((err / tol).max()), [int(i) for i in bad.nonzero()[0]])


def both(ops, q, k, v, dy, **kw):
    y, saved = ops.attention_forward(q, k, v, save=True, **kw)
    return dict(zip(("y",) + NAMES, (y,) + ops.attention_backward(dy, q, k, v, y, saved, **kw)))


def compare(ops, x, **kw):
    want = formula(*x, **kw)
    got = both(ops, *x, **kw)
    for name in want:
        check(name, got[name], want[name])
    alone = ops.attention_forward(*x[:3], **kw)                 # without keeping anything: the same bits
    assert torch.equal(alone, got["y"])
    return got, want


def slopes_of(H):
    return torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda") / H).float()


def documents_of(seed, B, n, count, padding=0):
    """documents one behind the other, of random lengths; `padding` places at the end belong to none"""
    g = torch.Generator()
    g.manual_seed(seed)
    ids = torch.full((B, n), -1, dtype=torch.int64)
    for b in range(B):
        live = n - padding
        cuts = sorted(torch.randint(0, live + 1, (count - 1,), generator=g).tolist())
        for i, (lo, hi) in enumerate(zip([0] + cuts, cuts + [live])):
            ids[b, lo:hi] = 3 * i
    return ids.cuda()


TERMS = [dict(), dict(cap=15.0), dict(slopes=True), dict(cap=5.0, slopes=True, scale=0.3)]


def terms(which, H):
    t = dict(TERMS[which])
    if t.get("slopes"):
        t["slopes"] = slopes_of(H)
    return t


# sizes around the tiles' (32 rows of an instruction, 64 keys of a tile, 128 rows of a workgroup), groups of every kind, odd head sizes
SHAPES = [(1, 1, 1, 1, 1, 1), (1, 1, 1, 1, 1, 64), (2, 3, 3, 2, 1, 8), (1, 31, 31, 1, 1, 64), (1, 32, 32, 2, 2, 128), (1, 33, 33, 1, 1, 16), (3, 17, 17, 4, 4, 64),
          (1, 63, 63, 3, 1, 72), (1, 64, 64, 7, 1, 40), (2, 65, 65, 6, 3, 96), (1, 127, 127, 2, 1, 128), (1, 128, 128, 8, 2, 64), (1, 129, 129, 5, 5, 33),
          (1, 200, 200, 12, 4, 80), (2, 255, 255, 2, 1, 127), (1, 257, 257, 9, 3, 128), (1, 515, 515, 4, 2, 65), (1, 700, 700, 4, 1, 128), (1, 1100, 1100, 2, 2, 64)]


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", SHAPES)
def test_causal(ops, shape, dtype):
    compare(ops, inputs(sum(shape), *shape, dtype), **terms(sum(shape) % 4, shape[3]))


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("d", [64, 128])
def test_every_kernel(ops, which, d, dtype):
    """the kernels for many rows and for few, with every combination of a score's terms"""
    for B, T, K, H, Hk in ((2, 150, 150, 4, 2), (2, 3, 200, 8, 2)):
        for causal in (True, False):
            compare(ops, inputs(which + T, B, T, K, H, Hk, d, dtype), causal=causal, **terms(which, H))


# new tokens behind those whose keys are there, and more queries than keys: the first ones see nothing
@pytest.mark.parametrize("T,K", [(1, 64), (5, 70), (40, 100), (130, 1000), (100, 40), (200, 1), (65, 64)])
@pytest.mark.parametrize("which", range(4))
def test_queries_and_keys_of_different_lengths(ops, T, K, which):
    x = inputs(T + K, 2, T, K, 4, 2, 64, torch.bfloat16)
    got, _ = compare(ops, x, **terms(which, 4))
    if T > K:
        assert not bool(got["y"][:, :T - K].any()) and not bool(got["dq"][:, :T - K].any())
    compare(ops, x, causal=False, **terms(which, 4))


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("B,K,H,Hk,d", [(1, 1, 8, 1, 128), (1, 31, 32, 1, 64), (2, 32, 4, 4, 128), (1, 33, 6, 2, 72), (3, 95, 8, 8, 64), (1, 1000, 40, 8, 128),
                                        (2, 4099, 8, 2, 128), (5, 513, 33, 3, 64), (1, 20000, 16, 2, 128), (1, 9000, 48, 1, 100), (70, 300, 16, 16, 64)])
def test_one_new_token(ops, B, K, H, Hk, d, dtype):
    for which in (0, 3):
        for causal in (True, False):
            kw = dict(causal=causal, **terms(which, H))
            q, k, v, _ = inputs(K + which, B, 1, K, H, Hk, d, dtype)
            check("y", ops.attention_forward(q, k, v, **kw), formula(q, k, v, **kw)["y"])


@pytest.mark.parametrize("T,K,H,Hk,d", [(256, 5000, 8, 2, 128), (100, 9000, 2, 1, 64), (40, 3001, 1, 1, 96)])
def test_few_rows_over_many_keys_are_split(ops, T, K, H, Hk, d):
    q, k, v, dy = inputs(K, 1, T, K, H, Hk, d, torch.bfloat16)
    compare(ops, (q, k, v, dy), slopes=slopes_of(H))


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("B,T,count,padding", [(1, 17, 3, 0), (2, 150, 4, 20), (1, 515, 7, 100), (2, 640, 2, 0), (1, 700, 40, 5)])
@pytest.mark.parametrize("which", [0, 3])
def test_documents(ops, B, T, count, padding, which, dtype):
    ids = documents_of(T, B, T, count, padding)
    for causal in (True, False):
        x = inputs(T, B, T, T, 6, 2, 72, dtype)
        got, _ = compare(ops, x, causal=causal, documents=ids, **terms(which, 6))
        none = ids < 0
        assert not any(bool(got[n][none].any()) for n in got)
    got32 = both(ops, *x, documents=ids.int(), causal=False, **terms(which, 6))
    assert all(torch.equal(got[n], got32[n]) for n in got)


@pytest.mark.parametrize("B,T,K,H,Hk,d,causal,count", [
    (1, 300, 1500, 2, 1, 64, True, 0), (1, 300, 1500, 2, 1, 128, True, 0), (9, 130, 130, 32, 32, 128, True, 0), (9, 130, 130, 32, 32, 128, True, 3),
    (17, 130, 130, 32, 32, 64, True, 0), (17, 130, 130, 32, 32, 64, False, 3), (1, 700, 700, 6, 2, 128, True, 0), (1, 700, 700, 6, 2, 128, False, 0),
    (1, 700, 700, 6, 2, 128, True, 5), (1, 1200, 1200, 8, 1, 64, True, 0), (1, 1200, 1200, 8, 1, 64, True, 4), (8, 1024, 1024, 16, 8, 128, True, 0),
    (2, 900, 900, 4, 2, 128, False, 12)])
def test_however_the_work_is_shared(ops, B, T, K, H, Hk, d, causal, count):
    """calls of every rule by which rows and keys are given to workgroups, in parts or not, dealt by the mask or not"""
    x = inputs(T + d, B, T, K, H, Hk, d, torch.bfloat16)
    kw = dict(causal=causal, cap=8.0)
    if count:
        kw["documents"] = documents_of(B + d, B, T, count, T // 9)
        if causal and B == 1:
            kw["prefix"] = torch.rand((B, T), generator=gen(3), device="cuda") < 0.2
    got, _ = compare(ops, x, **kw)
    again = both(ops, *x, **kw)
    assert all(torch.equal(got[n], again[n]) for n in got)


def test_documents_in_any_order(ops):
    """numbers that alternate, repeat far apart, are as large as they may be, or mean none"""
    T = 300
    ids = torch.stack([torch.arange(T) % 3, torch.arange(T) // 7 % 5, torch.tensor([2 ** 31 - 2, 2 ** 31 - 3, -1, 2 ** 31 - 1, 2 ** 40, -2 ** 40])[torch.arange(T) % 6]]).cuda()
    x = inputs(5, 3, T, T, 2, 1, 64, torch.float16)
    got, _ = compare(ops, x, documents=ids)
    assert not bool(got["y"][2, torch.arange(T, device="cuda") % 6 > 1].any())
    compare(ops, x, documents=ids, causal=False, cap=3.0)


def test_documents_named_by_other_tensors(ops):
    """the backward pass is told of the forward pass's documents by copies, pairs, other types and strides: the same gradients"""
    B, T = 2, 200
    x = inputs(5, B, T, T, 4, 2, 64, torch.bfloat16)
    ids = documents_of(1, B, T, 4, 15)
    prefix = torch.rand((B, T), generator=gen(2), device="cuda") < 0.3
    want = both(ops, *x, documents=ids, prefix=prefix)
    wide = torch.full((B, 2 * T), 9, dtype=torch.int32, device="cuda")
    wide[:, T:] = ids
    ways = (ids, ids.clone(), (ids, ids.clone()), wide[:, T:], (wide[:, T:], wide[:, T:].contiguous()))
    for one in ways:
        y, saved = ops.attention_forward(*x[:3], documents=one, prefix=prefix, save=True)
        for other in ways:
            got = ops.attention_backward(x[3], *x[:3], y, saved, documents=other, prefix=prefix.clone())
            assert all(torch.equal(g, want[n]) for n, g in zip(NAMES, got))
    with pytest.raises(Exception):
        ops.attention_backward(x[3], *x[:3], y, ops.attention_forward(*x[:3], save=True)[1], documents=ids)


@pytest.mark.parametrize("T,K,H,Hk", [(1, 700, 8, 2), (5, 300, 4, 2), (200, 700, 2, 1), (130, 64, 2, 2)])
def test_documents_of_queries_and_keys(ops, T, K, H, Hk):
    B = 4
    kid = documents_of(K, B, K, 3, 30)
    kid[2] = -1                                                 # a sequence without any key
    kid[3, K // 2:] = -1                                        # and one whose second half is not there
    qid = torch.zeros((B, T), dtype=torch.int64, device="cuda")
    qid[1, T // 2:] = 3
    if T > 3:
        qid[0, 2] = -1                                          # and a query of none
    for causal in (True, False):
        x = inputs(T, B, T, K, H, Hk, 64, torch.bfloat16)
        got, _ = compare(ops, x, documents=(qid, kid), causal=causal)
        assert not bool(got["y"][2].any()) and not bool(got["dk"][2].any())


@pytest.mark.parametrize("T,count,padding", [(40, 1, 0), (150, 2, 10), (515, 3, 60)])
@pytest.mark.parametrize("which", [0, 3])
def test_prefix(ops, T, count, padding, which):
    ids = documents_of(T, 2, T, count, padding)
    prefix = torch.zeros((2, T), dtype=torch.bool, device="cuda")
    for b in range(2):
        for doc in ids[b].unique():
            places = (ids[b] == doc).nonzero().flatten()
            prefix[b, places[:len(places) * (2 + b) // 5]] = True
    x = inputs(T, 2, T, T, 4, 2, 64, torch.float16)
    compare(ops, x, documents=ids, prefix=prefix, **terms(which, 4))
    compare(ops, x, prefix=prefix, **terms(which, 4))           # of one document
    g = torch.Generator()
    g.manual_seed(T)
    anywhere = (torch.rand((2, T), generator=g) < 0.1).cuda()   # and not only at its start
    compare(ops, x, documents=ids, prefix=anywhere.to(torch.uint8) * 7, **terms(which, 4))
    compare(ops, x, prefix=torch.ones_like(prefix), **terms(which, 4))


@pytest.mark.parametrize("T", [20, 300])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_places_of_no_document_may_hold_anything(ops, T, value):
    for causal in (True, False):
        ids = documents_of(T, 2, T, 2, T // 3)
        ids[1, 3:9] = -1
        x = inputs(T, 2, T, T, 4, 2, 128, torch.bfloat16)
        for t in x:
            t[ids < 0] = value
        y, saved = ops.attention_forward(*x[:3], documents=ids, causal=causal, save=True)
        got = dict(zip(NAMES, ops.attention_backward(x[3], *x[:3], y, saved, documents=ids, causal=causal)), y=y)
        want = formula(*x, documents=ids, causal=causal)
        for name in want:
            check(name, got[name], want[name])
            assert not bool(got[name][ids < 0].any())


@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (5, 7), (8, 0), (64, 8)])
@pytest.mark.parametrize("T", [6, 140])
def test_strides_and_alignment(ops, T, pad, shift):
    x = inputs(3, 2, T, T, 4, 2, 72, torch.float16, pad, shift)
    want = formula(*x)
    outs = [normal(gen(i), t.shape, torch.float16, 1.0, 5, 3) for i, t in enumerate((x[0], x[0], x[1], x[2]))]
    y, saved = ops.attention_forward(*x[:3], save=True, out=outs[0])
    assert y is outs[0]
    ops.attention_backward(x[3], *x[:3], y, saved, out=outs[1:])
    for name, t in zip(("y",) + NAMES, outs):
        check(name, t, want[name])
        assert bool(torch.isnan(t._base[:3]).all()) and bool(torch.isnan(t._base[3:].view(2, T, -1)[:, :, t.shape[2] * 72:]).all()), name


def test_one_projection_and_heads_first(ops):
    """queries, keys and values side by side, their gradients too; tensors laid out by heads; keys that all sequences share"""
    B, T, H, Hk, d = 2, 150, 4, 2, 64
    g = gen(9)
    both_ = torch.randn((B, T, H + 2 * Hk, d), generator=g, device="cuda").bfloat16()
    q, k, v = both_[:, :, :H], both_[:, :, H:H + Hk], both_[:, :, H + Hk:]
    dy = torch.randn((B, T, H, d), generator=g, device="cuda").bfloat16()
    want = formula(q, k, v, dy)
    y, saved = ops.attention_forward(q, k, v, save=True)
    grads = torch.full_like(both_, float("nan"))
    ops.attention_backward(dy, q, k, v, y, saved, out=(grads[:, :, :H], grads[:, :, H:H + Hk], grads[:, :, H + Hk:]))
    for name, t in zip(("y",) + NAMES, (y, grads[:, :, :H], grads[:, :, H:H + Hk], grads[:, :, H + Hk:])):
        check(name, t, want[name])
    by_head = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v, dy)]
    got = both(ops, *by_head)
    assert all(torch.equal(got[n], t) for n, t in zip(("y",) + NAMES, (y, grads[:, :, :H], grads[:, :, H:H + Hk], grads[:, :, H + Hk:])))
    shared = [q, k[:1].expand(B, -1, -1, -1), v[:1].expand(B, -1, -1, -1), dy]
    want = formula(*shared)
    for name, t in both(ops, *shared).items():
        check(name, t, want[name])


def test_a_result_among_the_rows_of_the_inputs(ops):
    """queries, keys, values and the result as columns of the same rows of memory"""
    B, T, H, d = 2, 90, 3, 40
    buf = torch.randn((B, T, 4 * H * d + 5), generator=gen(2), device="cuda").half()
    q, k, v, y = (buf[:, :, i * H * d:(i + 1) * H * d].unflatten(2, (H, d)) for i in range(4))
    rest = buf[:, :, 4 * H * d:].clone()
    want = formula(q, k, v)["y"]
    assert ops.attention_forward(q, k, v, out=y) is y
    check("y", y, want)
    assert torch.equal(buf[:, :, 4 * H * d:], rest)
    # a part of the tokens of a longer buffer, the others left as they were
    long = torch.full((B, 3 * T, H, d), 7.0, dtype=torch.float16, device="cuda")
    ops.attention_forward(q, k, v, out=long[:, T:2 * T])
    assert torch.equal(long[:, T:2 * T], y) and bool((long[:, :T] == 7).all()) and bool((long[:, 2 * T:] == 7).all())


def test_refusals(ops):
    from paper_2508_21613_amd.binding import ChmError
    q, k, v, dy = inputs(1, 2, 10, 12, 4, 2, 64, torch.bfloat16)
    ids = torch.zeros((2, 10), dtype=torch.int32, device="cuda")
    kid = torch.zeros((2, 12), dtype=torch.int32, device="cuda")
    slopes = slopes_of(4)
    bad = [((q.cpu(), k, v), {}), ((q, k.cpu(), v), {}), ((q, k, v.half()), {}), ((q.float(), k.float(), v.float()), {}), ((q[0], k, v), {}), ((q, k[:1], v), {}),
           ((q, k, v[:, :5]), {}), ((q[:, :, :3], k, v), {}), ((q[..., :32], k, v), {}), ((q.transpose(2, 3), k, v), {}), ((q, k[:, :, :0], v[:, :, :0]), {}),
           ((q, k, v), dict(scale=0)), ((q, k, v), dict(scale=-1)), ((q, k, v), dict(scale=float("nan"))), ((q, k, v), dict(cap=-1)), ((q, k, v), dict(cap=float("inf"))),
           ((q, k, v), dict(slopes=slopes[:3])), ((q, k, v), dict(slopes=slopes.double())), ((q, k, v), dict(slopes=slopes.cpu())), ((q, k, v), dict(slopes=[1.0] * 4)),
           ((q, k, v), dict(documents=ids)), ((q, k, v), dict(documents=(ids, ids))), ((q, k, v), dict(documents=(ids, kid.long()))), ((q, k, v), dict(documents=(ids.float(), kid.float()))),
           ((q, k, v), dict(documents=(ids, kid, kid))), ((q, k, v), dict(documents=(ids, None))), ((q, k, v), dict(prefix=kid)), ((q, k, v), dict(prefix=kid.bool(), causal=False)),
           ((q, k, v), dict(prefix=kid.bool()[:, :5])), ((q, k, v), dict(out=q)), ((q, k, v), dict(out=q[:1])), ((q, k, v), dict(out=q.half())), ((q, k, v), dict(out=k)),
           ((q, k, v), dict(out=torch.empty_like(q[:1]).expand(2, -1, -1, -1)))]
    for args, kw in bad:
        with pytest.raises(ChmError):
            ops.attention_forward(*args, **kw)
    big = torch.zeros((1, 3, 1, 136), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ChmError):
        ops.attention_forward(big, big, big)
    y, saved = ops.attention_forward(q, k, v, save=True)
    for args in ((dy[:, :5], q, k, v, y, saved), (dy.half(), q, k, v, y, saved), (dy, q, k, v, y[:1], saved), (dy, q, k, v, y, saved[:100]), (dy, q, k, v, y, None),
                 (dy, q, k, v, y, saved.view(torch.int8))):
        with pytest.raises(ChmError):
            ops.attention_backward(*args)
    for out in ((q, k, v), (torch.empty_like(q), torch.empty_like(k)), (torch.empty_like(q), torch.empty_like(k), v), (torch.empty_like(k), torch.empty_like(k), torch.empty_like(v))):
        with pytest.raises(ChmError):
            ops.attention_backward(dy, q, k, v, y, saved, out=out)


def test_inputs_that_require_a_gradient(ops):
    """the results are no part of autograd's graph: refused where the gradient would be lost, taken where the caller goes on by hand"""
    from paper_2508_21613_amd.binding import ChmError
    q, k, v, dy = inputs(1, 1, 20, 20, 2, 2, 64, torch.bfloat16)
    k.requires_grad_(True)
    with pytest.raises(ChmError):
        ops.attention_forward(q, k, v)
    y, saved = ops.attention_forward(q, k, v, save=True)
    assert not y.requires_grad and len(ops.attention_backward(dy, q, k, v, y, saved)) == 3
    with torch.no_grad():
        assert torch.equal(ops.attention_forward(q, k, v), y)
    with pytest.raises(ChmError):
        ops.attention_forward(q, k, v, save=True, slopes=slopes_of(2).requires_grad_(True))


def test_lengths_of_zero(ops):
    for B, T, K in ((0, 5, 5), (2, 0, 0), (2, 0, 70), (2, 70, 0), (2, 3, 0)):
        x = inputs(1, B, T, K, 4, 2, 64, torch.bfloat16)
        got = both(ops, *x, causal=False)
        for name, like in zip(("y",) + NAMES, (x[0], x[0], x[1], x[2])):
            assert got[name].shape == like.shape and not bool(got[name].any())


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("cap", [255.0, 257.0, 3000.0, 1e6, 1e30, 3e38])
@pytest.mark.parametrize("T,d", [(9, 64), (100, 128)])
def test_large_caps(ops, T, d, cap, dtype):
    """scores far below a cap keep their digits; a score of a tenth of the cap and more is there as well"""
    q, k, v, dy = inputs(T, 1, T, T, 4, 2, d, dtype)
    q[:, -1] *= 60.0
    compare(ops, (q, k, v, dy), cap=cap)
    one = ops.attention_forward(q[:, -1:], k, v, cap=cap)
    check("y", one, tuple(t[:, -1:] for t in formula(q, k, v, cap=cap)["y"]))


def test_scores_far_apart(ops):
    """maxima that grow from tile to tile by more than the exponential reaches, and scores beyond it either way"""
    B, T, H, d = 1, 400, 2, 64
    q, k, v, dy = inputs(2, B, T, T, H, H, d, torch.bfloat16)
    q[..., 0], k[..., 0] = 30.0, (torch.arange(T, device="cuda") * 0.5 - 100).bfloat16()[None, :, None]
    for sign in (1, -1):
        k[..., 0] *= sign
        for kw in (dict(), dict(cap=50.0)):
            compare(ops, (q, k, v, dy), **kw)


def test_infinities_and_nans_follow_the_formulas(ops):
    q, k, v, _ = inputs(4, 1, 70, 70, 1, 1, 64, torch.bfloat16)
    q[0, 40] = float("nan")
    y = ops.attention_forward(q, k, v)
    rows = torch.isnan(y[0, :, 0]).any(1)
    assert rows.nonzero().flatten().tolist() == [40] and bool(torch.isnan(y[0, 40]).all())
    q[0, 40] = 1.0
    k[0, 69] = float("inf")                                     # capped: a score of the cap, or less it
    q[0, 69] = 1.0
    y = ops.attention_forward(q, k, v, cap=8.0)
    assert bool(torch.isfinite(y).all())


def test_same_inputs_same_bits(ops):
    x = inputs(8, 1, 900, 900, 8, 2, 128, torch.bfloat16)
    ids = documents_of(1, 1, 900, 3, 9)
    first = both(ops, *x, documents=ids)
    for _ in range(3):
        again = both(ops, *x, documents=ids)
        assert all(torch.equal(first[n], again[n]) for n in first)


@pytest.mark.parametrize("which", [0, 3])
def test_gradients_against_differences(ops, which):
    """dy.y changes along a direction as the gradients say: central differences of the formula in 64 bits (off by step^2) against the kernels'
    gradients, whose errors' variances add up along the direction"""
    x = inputs(21, 1, 90, 90, 4, 2, 40, torch.float16)
    kw = terms(which, 4)
    got, want = both(ops, *x, **kw), formula(*x, **kw)

    def loss(t):
        return float((formula(*t, **kw)["y"][0] * x[3].double()).sum())

    # the 16-bit inputs are the middle; the formula takes them as 64-bit ones
    formula_dtype = torch.float64
    U[formula_dtype], TINY[formula_dtype] = 0.0, 0.0
    try:
        for i, name in enumerate(NAMES):
            step, g = 1e-4, gen(i)
            along = torch.randn(x[i].shape, generator=g, device="cuda", dtype=torch.float64)
            ends = []
            for sign in (1, -1):
                t = [a.double() for a in x[:3]]
                t[i] = t[i] + sign * step * along
                ends.append(loss(t))
            slope = (ends[0] - ends[1]) / (2 * step)
            here = float((got[name].double() * along).sum())
            sigma = float(((want[name][1] + (U[torch.float16] * want[name][0]) ** 2 / 3) * along ** 2).sum().sqrt())
            assert abs(here - slope) <= 6 * sigma + 1e-5 * abs(slope) + 1e-6, (name, here, slope, sigma)
    finally:
        del U[formula_dtype], TINY[formula_dtype]


def test_captured_and_replayed(ops):
    """a step in a graph, replayed with other inputs in the same places, eager work between the replays"""
    shape = (1, 300, 300, 4, 2, 64)
    ids = documents_of(3, 1, 300, 3, 20)
    place, others = inputs(1, *shape, torch.bfloat16), [inputs(s, *shape, torch.bfloat16) for s in (2, 3, 4)]
    tok = inputs(5, 2, 1, 5000, 8, 2, 128, torch.bfloat16)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both(ops, *place, documents=ids)
        ops.attention_forward(*tok[:3])
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(ops, *place, documents=ids)
        one = ops.attention_forward(*tok[:3])
    for x in others + others:
        for a, b in zip(place, x):
            a.copy_(b)
        tok[0].mul_(-1)
        graph.replay()
        want, want_one = both(ops, *x, documents=ids), ops.attention_forward(*tok[:3])
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want) and torch.equal(one, want_one)


def test_on_another_stream(ops):
    x = inputs(6, 1, 500, 500, 4, 2, 64, torch.bfloat16)
    want = both(ops, *x)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    y, saved = ops.attention_forward(*x[:3], save=True, stream=stream)
    got = (y,) + ops.attention_backward(x[3], *x[:3], y, saved, stream=stream.cuda_stream)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want.values()))


def test_offsets_beyond_32_bits(ops):
    """a cache of more than 2^31 elements, and tokens further apart than offsets of 31 bits reach within a tile"""
    K, Hk, d = 300000, 64, 128
    g = gen(1)
    k, v = (torch.empty((1, K, Hk, d), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g) for _ in range(2))
    q = normal(g, (1, 1, Hk, d), torch.bfloat16)
    y = ops.attention_forward(q, k, v)
    for h in (0, 31, 63):
        check("y", y[:, :, h:h + 1], formula(q[:, :, h:h + 1], k[:, :, h:h + 1], v[:, :, h:h + 1])["y"])
    wide = k.view(-1)[:(K // 8) * Hk * d * 8].view(1, 8, -1)[:, :, :Hk * d].unflatten(2, (Hk, d))          # 8 tokens 300 million elements apart
    y = ops.attention_forward(wide, wide, wide)
    check("y", y[:, :, :4], formula(wide[:, :, :4], wide[:, :, :4], wide[:, :, :4])["y"])


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("T,H,Hk,d", [(2, 1, 1, 64), (17, 4, 4, 64), (40, 6, 2, 128), (130, 4, 1, 80)])
def test_gradients_of_small_calls(ops, T, H, Hk, d, dtype):
    """there ds and p enter their products with what their rounding took: of the tensors' type's roundings are left the gradients' own and that of the forward pass's
    weights, which y brings into delta"""
    x = inputs(T, 1, T, T, H, Hk, d, dtype)
    got, want = both(ops, *x, cap=20.0), formula(*x, cap=20.0, kept=U[dtype])
    for name in NAMES:
        check(name, got[name], want[name])


@pytest.mark.parametrize("d,far", [(128, 17000000), (128, 8500000), (72, 8500000), (72, 8454650), (64, 17000000)])
def test_values_far_apart(ops, d, far):
    """values whose tokens lie millions of elements apart, others between them: the same bits as of values side by side"""
    T, H = 140, 2
    q, k, v, dy = inputs(d, 1, T, T, H, 1, d, torch.bfloat16)
    far = far // 8 * 8
    buf = torch.full((T * far,), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide = buf.view(1, T, far)[:, :, :d].unflatten(2, (1, d))
    wide.copy_(v)
    for kw in (dict(), dict(causal=False)):
        want, got = both(ops, q, k, v, dy, **kw), both(ops, q, k, wide, dy, **kw)
        assert all(torch.equal(got[n], want[n]) for n in want)


def quantum(monkeypatch, least):
    """what float16's rounding of p and ds takes at least, for formula()"""
    monkeypatch.setitem(TINY, torch.float16, least)


@pytest.mark.parametrize("std", [0.05, 1e-3, 2e-4, 5e-5])
@pytest.mark.parametrize("T,K,H,Hk,d,causal,cap", [(2048, 2048, 2, 2, 64, True, 0.0), (4096, 4096, 2, 1, 128, False, 0.0), (1500, 1500, 3, 1, 128, True, 20.0),
                                                   (300, 9000, 1, 1, 64, False, 500.0), (17, 17, 4, 4, 64, True, 0.0), (130, 3000, 2, 1, 72, True, 0.0)])
def test_gradients_of_small_dy_in_float16(ops, monkeypatch, T, K, H, Hk, d, causal, cap, std):
    """p and ds are taken 2^12 times as large: what rounding takes of them at least is 2^-37.  That of the forward pass's weights (2^-25, of weights whose sum is 1 and more)
    comes into delta, for which formula() grants y's rounding as well, which is kept: 2^-11 / sqrt(3) of an element of y of some 1 / sqrt(keys) is more
    than sqrt(keys) 2^-25 / sqrt(3) up to 2^14 keys.  As a whole, too, the error is within 1.1 standard deviations: of a hundred thousand elements and more that
    is 30 of its own standard deviations, and the few rows of the small calls, whose errors are alike, have 1.5."""
    x = inputs(T + d, 1, T, K, H, Hk, d, torch.float16)
    x[3].mul_(std / 0.3)
    quantum(monkeypatch, 2.0 ** -37)
    want = formula(*x, causal=causal, cap=cap)
    quantum(monkeypatch, 2.0 ** -25)
    got = both(ops, *x, causal=causal, cap=cap)
    for name in NAMES:
        check(name, got[name], want[name])
        value, var = want[name]
        own = torch.clamp(value.abs() * U[torch.float16], min=TINY[torch.float16]) ** 2 / 3
        assert float((got[name].double() - value).norm()) <= (1.1 if T > 1000 else 1.5) * float((var + own).sum().sqrt()), name


@pytest.mark.parametrize("std,scale", [(30.0, None), (1000.0, 0.002), (10000.0, 1e-4)])
@pytest.mark.parametrize("T,H,Hk,d,cap,which", [(50, 2, 1, 64, 0.0, 0), (700, 4, 2, 64, 0.0, 0), (700, 2, 2, 128, 0.0, 1), (1300, 2, 1, 128, 30.0, 0), (900, 2, 1, 80, 300.0, 1)])
def test_gradients_of_large_dy_in_float16(ops, monkeypatch, T, H, Hk, d, cap, which, std, scale):
    """ds of 8 and more are lifted by less than 2^12, those beyond 65,504 taken down: by what brings the largest that a row (for dk: a wavefront) has met to between 2^13
    and 2^15, so that rounding takes at least 2^-38 of that.  |ds| is at most |dy.v| + |dy.y|.  dy is a thousand times larger in a few rows than in the others, as
    loss scaling or single tokens make it.  Elements near the end of float16's range are left out."""
    x = inputs(T + d, 1, T, T, H, Hk, d, torch.float16)
    q, k, v, dy = x
    v.mul_(4.0)
    dy.mul_(std / 0.3 / 1000)
    dy[:, 1::37] *= 1000
    assert bool(torch.isfinite(dy).all())
    kw = dict(cap=cap, **({} if which == 0 else dict(slopes=slopes_of(H))), **({} if scale is None else dict(scale=scale)))
    quantum(monkeypatch, 2.0 ** -37)
    want = formula(*x, **kw)
    quantum(monkeypatch, 2.0 ** -25)
    largest = 2 * dy.double().norm(dim=3) * v.double().norm(dim=3).max()            # [1, T, H]
    assert float(largest.max()) > 65504 or std < 1000
    see, G = visible(1, T, T)[0].double(), H // Hk
    step = (kw.get("scale", d ** -0.5) * 2.0 ** -38) ** 2 / 3
    for h in range(H):
        want["dq"][1][0, :, h] += step * largest[0, :, h, None] ** 2 * (see @ k[0, :, h // G].double() ** 2)
        want["dk"][1][0, :, h // G] += step * largest.max() ** 2 * (see.T @ q[0, :, h].double() ** 2)
    got = both(ops, *x, **kw)
    for name in NAMES:
        inside = want[name][0].abs() < 60000
        assert float(inside.double().mean()) > 0.9
        check(name, got[name][inside], tuple(t[inside] for t in want[name]))


def test_results_of_more_words_than_a_join_counts(ops):
    """2^20 tokens of 128 heads of 128 over 64 keys: nothing is split, so nothing is joined.  All queries and all dy of a head are the same memory, so all rows of the results are
    the same bits; the first are those of a single token, up to the order of sums, of which the formula's errors hold."""
    T, K, H, d = 1 << 20, 64, 128, 128
    q, k, v, dy = inputs(7, 1, 1, K, H, H, d, torch.bfloat16)
    want = formula(q, k, v, dy, causal=False)
    many = [t.expand(1, T, H, d) for t in (q, dy)]
    y, saved = ops.attention_forward(many[0], k, v, causal=False, save=True)
    dq, dk, dv = ops.attention_backward(many[1], many[0], k, v, y, saved, causal=False)
    for name, t in (("y", y), ("dq", dq)):
        check(name, t[:, :1], want[name])
        check(name, t[:, -1:], want[name])
        for part in t[0].split(1 << 17):
            assert torch.equal(part, t[0, :1].expand(len(part), -1, -1)), name
    assert bool(torch.isfinite(dk).all()) and bool(torch.isfinite(dv).all())
    del y, saved, dq, part, t
    torch.cuda.empty_cache()


@pytest.mark.parametrize("B,T,K", [(0, 5, 5), (2, 0, 0), (2, 0, 70), (2, 70, 0), (2, 3, 0), (0, 0, 9)])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_documents_and_prefixes_of_lengths_of_zero(ops, B, T, K, index):
    q, k, v, dy = inputs(1, B, T, K, 4, 2, 64, torch.bfloat16)
    qid, kid = (torch.zeros((B, n), dtype=index, device="cuda") for n in (T, K))
    for kw in (dict(documents=(qid, kid)), dict(documents=(qid, kid), causal=False), dict(prefix=kid.bool()), dict(documents=(qid, kid), prefix=kid.bool())):
        got = both(ops, q, k, v, dy, **kw)
        for name, like in zip(("y",) + NAMES, (q, q, k, v)):
            assert got[name].shape == like.shape and not bool(got[name].any())


def test_gradients_that_would_be_lost(ops):
    """the backward pass is no part of autograd's graph either: a dy that carries one is refused; inputs and results that are leaves of the caller's are not"""
    from paper_2508_21613_amd.binding import ChmError
    q, k, v, dy = inputs(1, 1, 20, 20, 2, 2, 64, torch.bfloat16)
    want = both(ops, q, k, v, dy)
    y, saved = ops.attention_forward(q, k, v, save=True)
    for t in (q, k, v, y):
        t.requires_grad_(True)
    w = torch.ones((), device="cuda", requires_grad=True)
    with pytest.raises(ChmError):
        ops.attention_backward(dy * w.bfloat16(), q, k, v, y, saved)
    (y.float() * dy.float()).sum().backward()                   # y as the leaf of what follows
    got = ops.attention_backward(y.grad, q, k, v, y, saved)
    assert all(torch.equal(g, want[n]) for n, g in zip(NAMES, got))
    with torch.no_grad():
        got = ops.attention_backward(dy * w.bfloat16(), q, k, v, y, saved)
    assert all(torch.equal(g, want[n]) for n, g in zip(NAMES, got))


def test_tangents_are_refused(ops):
    """derivatives in forward mode have no call: they would come out as none, also where nothing is recorded"""
    import torch.autograd.forward_ad as forward_ad
    from paper_2508_21613_amd.binding import ChmError
    q, k, v, dy = inputs(1, 1, 20, 20, 2, 2, 64, torch.bfloat16)
    y, saved = ops.attention_forward(q, k, v, save=True)
    rope, pos = ops.Rotary(64), torch.arange(20, device="cuda")
    w = torch.randn((3, 96, 40), device="cuda").bfloat16()
    x, table = torch.randn((7, 40), device="cuda").bfloat16(), torch.randn((9, 40), device="cuda")
    kept = ops.ffn_forward(x, w[0], w[1], w[2].T.contiguous(), save=True)[1]
    calls = {"attention_forward": (lambda *t: ops.attention_forward(*t), (q, k, v)),
             "attention_forward, save": (lambda *t: ops.attention_forward(*t, save=True), (q, k, v)),
             "attention_backward": (lambda *t: ops.attention_backward(t[0], *t[1:5], saved), (dy, q, k, v, y)),
             "rotate": (lambda t: rope.rotate(t, pos), (q[0],)), "gradient": (lambda t: rope.gradient(t, pos), (dy[0],)),
             "ffn_forward": (lambda *t: ops.ffn_forward(*t), (x, w[0], w[1], w[2].T.contiguous())),
             "ffn_forward, save": (lambda *t: ops.ffn_forward(*t, save=True), (x, w[0], w[1], w[2].T.contiguous())),
             "embedding_lookup": (lambda t: ops.embedding_lookup(pos[:5], t), (table,)),
             "embedding_gradient": (lambda t: ops.embedding_gradient(t, pos[:9], rows=20), (table,)),
             "ffn_backward": (lambda *t: ops.ffn_backward(*t, kept), (x, x, w[0], w[1], w[2].T.contiguous())),
             "Gradients": (lambda *t: ops.Gradients(t).close(), (table, x))}
    for name, (call, args) in calls.items():
        call(*args)
        with forward_ad.dual_level():
            call(*args)
            for i in range(len(args)):
                for recorded in (True, False):
                    with torch.set_grad_enabled(recorded), pytest.raises(ChmError):
                        call(*[forward_ad.make_dual(t, torch.ones_like(t)) if i == j else t for j, t in enumerate(args)])
        call(*args)


@pytest.mark.parametrize("T,d", [(20, 128), (300, 64), (900, 128)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_places_of_no_document_say_nothing_of_float16s_range(ops, monkeypatch, T, d, value):
    """what is taken from ds's lift goes by the pairs that are seen: the same gradients, bit by bit, as with zeros in the places of no document, for a dy that passes the range as for
    one that does not"""
    ids = documents_of(T, 2, T, 2, T // 3)
    ids[1, 3:9] = -1
    for std in (0.01, 3000.0):
        x = inputs(T, 2, T, T, 4, 2, d, torch.float16)
        x[3].mul_(std / 0.3)
        got = []
        for fill in (0.0, value):
            for t in x:
                t[ids < 0] = fill
            for causal in (True, False):
                got.append(both(ops, *x, documents=ids, causal=causal, scale=0.001))
        for want, other in zip(got[:2], got[2:]):
            for name in want:
                assert bool(torch.isfinite(other[name]).all()) or (std > 1000 and name == "dv")
                assert torch.equal(want[name].nan_to_num(7.0), other[name].nan_to_num(7.0)), name


def test_float16_captured_with_other_ranges(ops):
    """a captured backward pass takes as much of the lift as the dy at hand wants, at every replay"""
    x = inputs(11, 1, 400, 400, 4, 2, 128, torch.float16)
    dy = x[3].clone()
    y, saved = ops.attention_forward(*x[:3], save=True, scale=0.001)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ops.attention_backward(dy, *x[:3], y, saved, scale=0.001)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops.attention_backward(dy, *x[:3], y, saved, scale=0.001)
    for factor in (1.0, 1e4, 1e-3, 3e3, 1.0):
        dy.copy_(x[3] * factor)
        graph.replay()
        want = ops.attention_backward(dy, *x[:3], y, saved, scale=0.001)
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want)) and bool(torch.isfinite(got[0]).all())
