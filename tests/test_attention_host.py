"""What attention's and the rotary positions' entry points answer without a GPU: sizes of workspaces, kernels, refusals.  Nothing here is launched: every call
is refused, or has nothing to do."""
import ctypes as C
import math

import pytest

from paper_2508_21613_amd import binding as B

BASE = 1 << 40                     # addresses that nothing is read from


def _tensor(at, tokens, heads, dim, batch=1, pad=0):
    """address and strides of [batch, tokens, heads, dim] with `pad` elements behind every token, and the address behind it"""
    token = heads * dim + pad
    return at, (tokens * token, token, dim), at + batch * tokens * token * 2 + 256


def _attention(batch=2, tokens=100, keys=100, heads=8, kv_heads=2, dim=64, pad=0, **kw):
    at = BASE
    q, qs, at = _tensor(at, tokens, heads, dim, batch, pad)
    k, ks, at = _tensor(at, keys, kv_heads, dim, batch, pad)
    v, vs, at = _tensor(at, keys, kv_heads, dim, batch, pad)
    a = B.Attention(1, 1, batch, tokens, keys, heads, kv_heads, dim, q, k, v, qs, ks, vs, 0.125, 0.0)
    for name, value in kw.items():
        setattr(a, name, B.Strides(*value) if name.endswith("stride") else value)
    return a


def _gradients(a, at=BASE + (1 << 36), **kw):
    B_, T, K, H, Hk, d = a.batch, a.tokens, a.keys, a.heads, a.kv_heads, a.dim
    g = B.AttentionGradients()
    for name, n, h in (("dy", T, H), ("y", T, H), ("dq", T, H), ("dk", K, Hk), ("dv", K, Hk)):
        p, s, at = _tensor(at, n, h, d, B_)
        setattr(g, name, p)
        setattr(g, name + "_stride", B.Strides(*s))
    for name, value in kw.items():
        setattr(g, name, B.Strides(*value) if name.endswith("stride") else value)
    return g


def _sizes(a, g=None):
    out = [C.c_uint64() for _ in range(3)]
    rc = B.lib().chm_attention_sizes(a, g, *out)
    return rc, [int(v.value) for v in out]


def _kernels(a, g=None):
    k = B.AttentionKernels()
    return B.lib().chm_attention_selection(a, g, k), {n: getattr(k, n) for n, _ in k._fields_}


def test_sizes():
    a = _attention()
    rc, (saved, forward, backward) = _sizes(a, _gradients(a))
    rows = 448                                                             # 100 x 4, whole tiles of 64
    assert rc == B.OK and saved == 2 * 2 * rows * 4 + 2 * 100 * 8 * 64 * 2 and forward == 0
    assert backward >= 2 * 2 * rows // 32 * 640
    assert _sizes(a)[1][2] == 0
    odd = _attention(dim=63)
    assert _sizes(odd)[1][1] >= 2 * 100 * (8 + 2 + 2) * 64 * 2             # all three packed, to rows of 64
    one = _attention(pad=3, batch=1)
    assert _sizes(one)[1][1] >= 100 * (8 + 2 + 2) * 64 * 2
    docs = _attention(index_bits=32, q_documents=BASE >> 1, k_documents=BASE >> 1, ld_q_documents=100, ld_k_documents=100)
    assert _sizes(docs)[1][1] >= 2 * 128 * 4 and _sizes(docs)[1][0] >= saved + 2 * 128 * 4
    docs.saved = BASE >> 2
    assert _sizes(docs)[1][1] == 0                                         # what the tokens' documents are lies there
    for empty in (_attention(batch=0), _attention(tokens=0), _attention(keys=0), _attention(tokens=0, keys=0)):
        assert _sizes(empty, _gradients(empty))[0] == B.OK


def test_which_kernels():
    assert _kernels(_attention(tokens=1, keys=32768, heads=32, kv_heads=8, dim=128, batch=8))[1] == dict(
        few=1, dim=128, packed=0, forward_rows=32, dq_rows=0, dkdv_keys=0, forward_splits=4, dkdv_splits=1, dkdv_shared=0, fine=0)
    a = _attention(tokens=8192, keys=8192, heads=32, kv_heads=8, dim=128, batch=1)
    k = _kernels(a, _gradients(a))[1]
    assert (k["few"], k["packed"], k["forward_rows"], k["dq_rows"], k["dkdv_keys"], k["forward_splits"], k["dkdv_splits"]) == (0, 0, 128, 128, 128, 1, 2)
    assert _kernels(_attention(tokens=8, heads=8, kv_heads=2))[1]["few"] == 1 and _kernels(_attention(tokens=9, heads=8, kv_heads=2))[1]["few"] == 0
    assert _kernels(_attention(tokens=256, keys=32768, heads=32, kv_heads=8, dim=128, batch=1))[1]["forward_splits"] == 8
    assert _kernels(_attention(dim=65))[1]["packed"] == 7 and _kernels(_attention(dim=72))[1] == dict(_kernels(_attention(dim=72))[1], packed=0, dim=128)
    assert _kernels(_attention(k=BASE + 2))[1]["packed"] == 2
    # tokens so far apart that 64 of them are beyond offsets of 31 bits
    assert _kernels(_attention(batch=1, v_stride=(0, 1 << 25, 64)))[1]["packed"] == 4
    assert _kernels(_attention(batch=1, v_stride=(0, 1 << 24, 64)))[1]["packed"] == 0


def test_gradients_by_twice_the_products():
    for kw, want in ((dict(batch=1, tokens=17, keys=17, heads=4, kv_heads=4, dim=64), 1), (dict(batch=1, tokens=256, keys=256, heads=32, kv_heads=8, dim=128), 1),
                     (dict(batch=1, tokens=257, keys=257, heads=32, kv_heads=8, dim=128), 0), (dict(batch=1, tokens=1, keys=100000, heads=32, kv_heads=8, dim=64, causal=0), 1)):
        a = _attention(**kw)
        k = _kernels(a, _gradients(a))[1]
        assert k["fine"] == want and (k["dq_rows"] == 64 or not want)


@pytest.mark.parametrize("kw,want", [
    # (rows of the forward pass and of dq, keys, parts of the forward pass and of dk and dv, dealt)
    (dict(batch=1, tokens=300, keys=1500, heads=2, kv_heads=1, dim=64), (64, 64, 64, 3, 1, 0)),
    (dict(batch=1, tokens=300, keys=1500, heads=2, kv_heads=1, dim=128), (64, 64, 128, 3, 5, 1)),
    (dict(batch=9, tokens=130, keys=130, heads=32, kv_heads=32, dim=128), (128, 128, 128, 1, 1, 0)),
    (dict(batch=9, tokens=130, keys=130, heads=32, kv_heads=32, dim=128, documents=True), (128, 128, 128, 1, 1, 1)),
    (dict(batch=17, tokens=130, keys=130, heads=32, kv_heads=32, dim=64), (64, 128, 64, 1, 1, 0)),
    (dict(batch=17, tokens=130, keys=130, heads=32, kv_heads=32, dim=64, documents=True), (64, 128, 64, 1, 1, 1)),
    (dict(batch=1, tokens=700, keys=700, heads=6, kv_heads=2, dim=128), (64, 64, 128, 1, 16, 1)),
    (dict(batch=1, tokens=700, keys=700, heads=6, kv_heads=2, dim=128, causal=0), (64, 64, 128, 1, 8, 0)),
    (dict(batch=1, tokens=1200, keys=1200, heads=8, kv_heads=1, dim=64), (64, 64, 64, 2, 9, 1)),
    (dict(batch=8, tokens=1024, keys=1024, heads=16, kv_heads=8, dim=128), (128, 128, 128, 1, 2, 0)),
    (dict(batch=1, tokens=100, keys=131073, heads=1, kv_heads=1, dim=128), (128, 64, 128, 16, 1, 0))])
def test_how_work_is_shared(kw, want):
    documents = kw.pop("documents", False)
    a = _attention(**kw)
    if documents:
        a.index_bits, a.q_documents, a.k_documents, a.ld_q_documents, a.ld_k_documents = 32, BASE >> 1, BASE >> 1, a.tokens, a.keys
    k = _kernels(a, _gradients(a))[1]
    assert tuple(k[n] for n in ("forward_rows", "dq_rows", "dkdv_keys", "forward_splits", "dkdv_splits", "dkdv_shared")) == want


@pytest.mark.parametrize("kw", [
    dict(dtype=0), dict(dtype=3), dict(batch=-1), dict(tokens=-1), dict(keys=-1), dict(tokens=(1 << 30) + 1), dict(keys=(1 << 30) + 1), dict(heads=0),
    dict(kv_heads=0), dict(kv_heads=3), dict(kv_heads=16), dict(dim=0), dict(dim=129), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=2e30), dict(cap=1e-32),
    dict(scale=math.nan), dict(cap=-1.0), dict(cap=math.nan), dict(cap=math.inf), dict(q=BASE + 1), dict(k=BASE + 1), dict(v=BASE + 1),
    dict(saved=BASE + 8), dict(slopes=BASE + 2), dict(q_stride=(-1, 512, 64)), dict(k_stride=(0, -5, 64)), dict(v_stride=(0, 0, 1 << 61)),
    dict(q_documents=BASE, index_bits=32), dict(k_documents=BASE, index_bits=32), dict(q_documents=BASE, k_documents=BASE, index_bits=16),
    dict(q_documents=BASE + 4, k_documents=BASE, index_bits=64), dict(prefix=BASE, causal=0), dict(tokens=1 << 30, heads=16, kv_heads=1),
    dict(q_documents=BASE, k_documents=BASE, index_bits=32, ld_k_documents=-1), dict(prefix=BASE, ld_prefix=-100)])
def test_refused_descriptions(kw):
    a = _attention()
    for name, value in kw.items():
        setattr(a, name, B.Strides(*value) if name.endswith("stride") else value)
    assert _sizes(a)[0] == B.ERR_ARG and _kernels(a)[0] == B.ERR_ARG
    out = B.Strides(51200, 512, 64)
    assert B.lib().chm_attention_forward(a, BASE + (1 << 37), out, BASE + (1 << 38), 1 << 30, None) == B.ERR_ARG
    a.saved = a.saved or BASE + (1 << 35)
    assert B.lib().chm_attention_backward(a, _gradients(_attention()), BASE + (1 << 38), 1 << 30, None) == B.ERR_ARG


def _forward(a, y=BASE + (1 << 37), stride=None, scratch=BASE + (1 << 38), have=1 << 34):
    return B.lib().chm_attention_forward(a, y, B.Strides(*(stride or (a.tokens * a.heads * a.dim, a.heads * a.dim, a.dim))), scratch, have, None)


def _backward(a, g, scratch=BASE + (1 << 38), have=1 << 34):
    return B.lib().chm_attention_backward(a, g, scratch, have, None)


def test_refused_calls():
    a = _attention(pad=3)                                                  # has to be packed: wants scratch
    assert _forward(a, y=0) == B.ERR_ARG and _forward(a, y=BASE + (1 << 37) + 1) == B.ERR_ARG and _forward(a, scratch=0) == B.ERR_ARG
    assert _forward(a, scratch=BASE + (1 << 38) + 8) == B.ERR_ARG and _forward(a, have=100) == B.ERR_LIMIT
    assert _forward(a, stride=(51200, -512, 64)) == B.ERR_ARG and B.lib().chm_attention_forward(None, BASE, B.Strides(1, 1, 1), BASE, 0, None) == B.ERR_ARG
    for name in ("q", "k", "v"):
        b = _attention(pad=3, **{name: 0})
        assert _forward(b) == B.ERR_ARG
    # results over inputs, over themselves, scratch or saved over either
    for at in (a.q, a.k, a.v, a.q + 2 * 8 * 64, a.v + 2):
        assert _forward(a, y=at) == B.ERR_ARG
    assert _forward(a, stride=(0, 512, 64)) == B.ERR_ARG and _forward(a, stride=(51200, 500, 64)) == B.ERR_ARG and _forward(a, stride=(51200, 512, 32)) == B.ERR_ARG
    assert _forward(a, scratch=a.k) == B.ERR_ARG and _forward(a, scratch=BASE + (1 << 37) + 4096) == B.ERR_ARG
    assert _forward(_attention(saved=BASE + 4096)) == B.ERR_ARG and _forward(_attention(saved=BASE + (1 << 37))) == B.ERR_ARG
    assert _forward(_attention(slopes=BASE + (1 << 37))) == B.ERR_ARG
    docs = dict(index_bits=64, q_documents=BASE + (1 << 37) + 128, k_documents=BASE + (1 << 39), ld_q_documents=100, ld_k_documents=100)
    assert _forward(_attention(**docs)) == B.ERR_ARG
    assert _forward(_attention(prefix=BASE + (1 << 37) + 51200 * 4 - 1, ld_prefix=100)) == B.ERR_ARG


def test_refused_backward_calls():
    a = _attention(saved=BASE + (1 << 35))
    for name in ("dy", "y", "dq", "dk", "dv"):
        assert _backward(a, _gradients(a, **{name: 0})) == B.ERR_ARG
        assert _backward(a, _gradients(a, **{name: BASE + (1 << 36) + 1})) == B.ERR_ARG
        assert _backward(a, _gradients(a, **{name + "_stride": (1, -1, 1)})) == B.ERR_ARG
    assert _backward(_attention(), _gradients(a)) == B.ERR_ARG             # nothing saved
    assert _backward(a, None) == B.ERR_ARG and _backward(a, _gradients(a), have=64) == B.ERR_LIMIT and _backward(a, _gradients(a), scratch=0) == B.ERR_ARG
    g = _gradients(a)
    for result in ("dq", "dk", "dv"):
        for other in (a.q, a.k, a.v, g.dy, g.y, a.saved, g.dq if result != "dq" else g.dk):
            assert _backward(a, _gradients(a, **{result: other})) == B.ERR_ARG
        assert _backward(a, _gradients(a, **{result + "_stride": (0, 512, 64)})) == B.ERR_ARG
    assert _backward(a, g, scratch=a.saved) == B.ERR_ARG


def test_nothing_to_do():
    for a in (_attention(batch=0), _attention(tokens=0)):
        assert _forward(a, scratch=0, have=0) == B.OK
    a = _attention(batch=0)
    assert _backward(a, _gradients(a), scratch=0, have=0) == B.OK
    a = _attention(tokens=0, keys=0)
    assert _backward(a, _gradients(a), scratch=0, have=0) == B.OK


def test_results_among_the_rows_of_inputs():
    """queries, keys, values and the result as columns of the same rows of memory: one element too far to the left is refused"""
    H, d, T = 8, 64, 100
    side = 3 * H * d + 3
    stride = (T * side, side, d)
    a = _attention(kv_heads=8, q=BASE, k=BASE, v=BASE + H * d * 2, q_stride=stride, k_stride=stride, v_stride=stride)
    for y in (BASE + 4 * H * d - 2, BASE + 2 * side - 2 * H * d + 2, BASE, BASE + 2):
        assert _forward(a, y=y, stride=stride) == B.ERR_ARG


# ---------------------------------------------------------------------------------------------- rotary
def _rotary(pairs=8, **kw):
    f = (C.c_double * 128)(*[1.0 / (i + 1) for i in range(128)])
    axis = (C.c_int32 * 128)()
    r = B.RotaryTurn(1, 64, 0, 1, 10, 4, 16, pairs, BASE, BASE + (1 << 30), 64, 16, 64, 16, BASE + (1 << 31), 10, 1, C.addressof(f), C.addressof(axis))
    keep = (f, axis)
    for name, value in kw.items():
        setattr(r, name, value)
    return r, keep


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(dtype=-1), dict(index_bits=16), dict(pairing=2), dict(axes=0), dict(tokens=-1), dict(heads=-1), dict(pairs=0), dict(pairs=129, head_dim=300),
    dict(pairs=9), dict(head_dim=(1 << 20) + 1), dict(x=BASE + 1), dict(out=BASE + 1), dict(positions=BASE + 4), dict(x=0), dict(out=0), dict(positions=0),
    dict(frequencies=0), dict(x_token=-1), dict(out_head=-16), dict(positions_token=-1), dict(positions_axis=-1), dict(out_token=0), dict(out_token=48), dict(out_head=8),
    dict(out=BASE + 2), dict(out=BASE + 32), dict(out=BASE, out_token=64, out_head=16, x_head=32, x_token=128), dict(out=BASE + (1 << 31) + 8)])
def test_rotary_refusals(kw):
    r, keep = _rotary(**kw)
    assert B.lib().chm_rotary_turn(r, 0, None) == B.ERR_ARG


def test_rotary_refuses_axes_and_frequencies():
    r, (f, axis) = _rotary()
    axis[3] = 1
    assert B.lib().chm_rotary_turn(r, 0, None) == B.ERR_ARG
    axis[3] = -1
    assert B.lib().chm_rotary_turn(r, 0, None) == B.ERR_ARG
    axis[3] = 0
    for bad in (math.inf, math.nan):
        f[7] = bad
        assert B.lib().chm_rotary_turn(r, 0, None) == B.ERR_ARG
    f[7] = 1.0
    assert B.lib().chm_rotary_turn(None, 0, None) == B.ERR_ARG
    for nothing in (dict(tokens=0), dict(heads=0)):
        r, keep = _rotary(x=0, out=0, positions=0, **nothing)
        assert B.lib().chm_rotary_turn(r, 0, None) == B.OK


def test_rotary_descriptions():
    from paper_2508_21613_amd import operators as ops
    r = ops.Rotary(128, [16, 24, 24], base=5e5)
    assert (r.pairs, r.axes) == (64, 3) and list(r._axis) == [0] * 16 + [1] * 24 + [2] * 24 and r._frequencies[32] == 5e5 ** -0.5
    assert ops.Rotary(80).pairs == 40 and ops.Rotary(80, frequencies=[0.5, 0.25]).pairs == 2 and ops.Rotary(8, axes=[1, 0]).axes == 2
    for args, kw in (((1,), {}), ((128.0,), {}), ((128,), dict(sections=[40, 25])), ((128,), dict(sections=[])), ((128,), dict(sections=[-1, 3])), ((128,), dict(pairing="thirds")),
                     ((128,), dict(sections=[8], axes=[0])), ((128,), dict(axes=[])), ((128,), dict(axes=[256])), ((128,), dict(frequencies=[math.nan])),
                     ((128,), dict(sections=[2], frequencies=[1.0])), ((128,), dict(base=0.0)), ((300,), {})):
        with pytest.raises(B.ChmError):
            ops.Rotary(*args, **kw)


def test_tensors_that_are_not_on_the_gpu_are_refused():
    import torch
    from paper_2508_21613_amd import operators as ops
    x = torch.zeros((1, 4, 2, 8), dtype=torch.bfloat16)
    with pytest.raises(B.ChmError):
        ops.attention_forward(x, x, x)
    with pytest.raises(B.ChmError):
        ops.Rotary(8).rotate(x[0], torch.arange(4))
    for bad in (x[0], x.float(), None, "x"):
        with pytest.raises(B.ChmError):
            ops.attention_forward(bad, x, x)


def test_every_row_of_a_load_is_within_reach():
    """offsets within a load of whole rows count 31 bits: 64 rows of every input, 128 of the values where the gradients' kernels take 128 keys at a time"""
    at = ((1 << 31) - 256) // 2 - 128                                      # elements
    for dim, rows in ((64, 64), (65, 128), (72, 128), (128, 128)):
        kw = dict(batch=1, tokens=200, keys=200, heads=2, kv_heads=1, dim=dim)
        token = at // (rows - 1) // 8 * 8
        odd = 7 if dim % 8 else 0                                          # every input is packed: its rows are no whole words
        for far, forward, backward in ((token, 0, 0), (token + 8, 4 if rows == 64 else 0, 4), (17000000 // 8 * 8, 4 if rows == 64 and token < 17000000 else 0, 4 if token < 17000000 else 0)):
            a = _attention(**dict(kw, v_stride=(0, far, dim)))
            assert _kernels(a)[1]["packed"] == (odd or forward)
            assert _kernels(a, _gradients(a))[1]["packed"] == ((odd and 15) or backward)
    # keys are taken 64 at a time, or row by row
    a = _attention(batch=1, tokens=200, keys=200, heads=2, kv_heads=1, dim=128, k_stride=(0, 17000000, 128))
    assert _kernels(a, _gradients(a))[1]["packed"] == 0
    # strides of which no 64 can be counted
    for stride in (1 << 30, 1 << 31, 1 << 40, (1 << 58) // 200):
        for name in ("q_stride", "k_stride", "v_stride"):
            a = _attention(batch=1, tokens=200, keys=200, heads=2, kv_heads=1, dim=128, **{name: (0, stride, 128)})
            assert _kernels(a)[1]["packed"] == {"q_stride": 1, "k_stride": 2, "v_stride": 4}[name]
    a = _attention(batch=1, tokens=200, keys=200, heads=2, kv_heads=1, dim=128, q_stride=(0, 256, (1 << 58) // 2))
    assert _kernels(a)[1]["packed"] == 1


@pytest.mark.parametrize("kw", [dict(batch=1, tokens=1 << 20, keys=64, heads=128, kv_heads=128, dim=128), dict(batch=64, tokens=65536, keys=65536, heads=64, kv_heads=64, dim=128),
                                dict(batch=1, tokens=64, keys=1 << 22, heads=64, kv_heads=64, dim=64)])
def test_unsplit_calls_need_no_join(kw):
    """results of more words than the join's threads can count are refused only where there is a join"""
    a = _attention(**kw)
    g = _gradients(a, at=BASE + (1 << 46))
    rc, (saved, forward, backward) = _sizes(a, g)
    assert rc == B.OK and saved > 0 and backward > 0
    k = _kernels(a, g)[1]
    words = [a.batch * n * h * (a.dim // 4) for n, h in ((a.tokens, a.heads), (a.keys, a.kv_heads))]
    assert max(words) >= 1 << 32
    for splits, n in ((k["forward_splits"], words[0]), (k["dkdv_splits"], words[1])):
        assert splits == 1 or n < 1 << 32


@pytest.mark.parametrize("batch,tokens", [(1 << 18, 1), (1 << 17, 1), (1 << 16, 32), (65535, 32)])
def test_few_rows_of_very_many_heads_are_not_split(batch, tokens):
    """where two parts of every head, or their join, would be more than a grid counts"""
    a = _attention(batch=batch, tokens=tokens, keys=2048, heads=63, kv_heads=63, dim=128, causal=0)
    rc, k = _kernels(a)
    assert rc == B.OK and k["few"] == 1 and batch * 63 * k["forward_splits"] * 256 < 1 << 32
    assert k["forward_splits"] == 1 or batch * 63 * tokens * 32 < 1 << 32


@pytest.mark.parametrize("bits", [32, 64])
def test_documents_of_nothing(bits):
    """a tensor of no elements has no address: documents are asked for where there are queries and keys"""
    for kw in (dict(tokens=0), dict(keys=0), dict(tokens=0, keys=0), dict(batch=0)):
        for q, k in ((0, BASE >> 1), (BASE >> 1, 0), (0, 0), (BASE >> 1, BASE >> 2)):
            a = _attention(**kw, index_bits=bits, q_documents=q, k_documents=k, ld_q_documents=100, ld_k_documents=100, prefix=BASE >> 3, ld_prefix=100)
            g = _gradients(a)
            rc, (saved, forward, backward) = _sizes(a, g)
            assert rc == B.OK and _kernels(a, g)[0] == B.OK
            assert (saved, forward, backward) == tuple(_sizes(_attention(**kw), _gradients(_attention(**kw)))[1])       # nothing is kept of them
            if a.batch == 0 or a.tokens == 0:
                assert _forward(a, scratch=0, have=0) == B.OK
            if a.batch == 0 or (a.tokens == 0 and a.keys == 0):
                assert _backward(a, g, scratch=0, have=0) == B.OK
    for q, k in ((0, BASE >> 1), (BASE >> 1, 0)):
        assert _sizes(_attention(index_bits=bits, q_documents=q, k_documents=k, ld_q_documents=100, ld_k_documents=100))[0] == B.ERR_ARG


def test_what_carries_a_derivative_is_told():
    import torch
    import torch.autograd.forward_ad as forward_ad
    from paper_2508_21613_amd import operators as ops
    a, w = torch.ones(3), torch.ones(3, requires_grad=True)
    ops._unrecorded(a, a)
    for t in (w, w * 2):
        with pytest.raises(B.ChmError):
            ops._unrecorded(a, t)
        ops._unrecorded(a, t, kept=True)
        with torch.no_grad():
            ops._unrecorded(a, t)
    with forward_ad.dual_level():
        ops._unrecorded(a)
        dual = forward_ad.make_dual(a, torch.ones(3))
        for t in (dual, dual.view(1, 3), dual * 2):
            for kept in (False, True):
                with pytest.raises(B.ChmError):
                    ops._unrecorded(a, t, kept=kept)
                with torch.no_grad(), pytest.raises(B.ChmError):
                    ops._unrecorded(a, t, kept=kept)
    ops._unrecorded(a)


@pytest.mark.parametrize("far", [1 << 62, (1 << 63) - 8, 1 << 60])
def test_strides_beyond_what_bytes_can_count(far):
    """their ends wrap in 64 bits: refused, not compared with other tensors' places"""
    for name in ("x_token", "x_head", "out_token", "out_head", "positions_axis", "positions_token"):
        r, keep = _rotary(dtype=0, axes=2, **{name: far})
        assert B.lib().chm_rotary_turn(r, 0, None) == B.ERR_ARG, name
    docs = dict(index_bits=64, q_documents=BASE >> 1, k_documents=BASE >> 2, ld_q_documents=100, ld_k_documents=100, prefix=BASE >> 3, ld_prefix=100)
    assert _sizes(_attention(**docs))[0] == B.OK
    for name in ("ld_q_documents", "ld_k_documents", "ld_prefix"):
        assert _sizes(_attention(**dict(docs, **{name: far})))[0] == B.ERR_ARG, name
        one = _attention(batch=1, **dict(docs, **{name: far}))               # says nothing there
        assert _sizes(one)[0] == B.OK
        assert _forward(one, scratch=0) == B.ERR_ARG
    for nothing in (dict(tokens=1, x_token=far, out_token=far, positions_token=far), dict(heads=1, x_head=far, out_head=far)):
        r, keep = _rotary(**nothing, x=0)                                   # nor of a single token or head: refused for x
        assert B.lib().chm_rotary_turn(r, 0, None) == B.ERR_ARG
