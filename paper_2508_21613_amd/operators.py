"""Operators of a pipeline stage's training step, over torch tensors: the calls of include/chm_operators.h.

The gated feed-forward block forward and backward, the embedding's lookup and gradient, rotary positions, attention forward and backward, the
global gradient norm with clipping.
As everywhere in this package torch provides device memory and streams; every value is computed by the library's HIP kernels, and
without a usable GPU the calls fail.  A call works on the current stream, or on `stream`; scratch and results that the caller does
not hand in are allocated on that stream.  Inputs must be ready there, as with any torch call.  Results must not lie over inputs or each
other (ffn_forward's may lie over x).  Wrong arguments raise binding.ChmError with the library's code.

Results are no part of autograd's graph; the gradients are calls of their own.  While torch records gradients, inputs that require one are
taken only where the caller asks for what the gradient's call wants (ffn_forward and attention_forward with save=True): anything else would lose it without a word.
So would the backward calls' gradients with respect to their dy: those of attention and the rotary positions refuse one that requires a gradient.  Inputs
with tangents of torch.autograd.forward_ad are refused.
"""
import ctypes as C
import math

import torch
from torch.autograd import forward_ad

from . import binding as B

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
INDEX_BITS = {torch.int32: 32, torch.int64: 64}
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}


def _need(ok, what):
    if not ok:
        raise B.ChmError(B.ERR_ARG, what)


def _matrix(name, t, rows=None, cols=None, dtype=None, device=None):
    """checks a row-major matrix (unit stride along rows) and returns the elements from one row to the next; device: an index"""
    if not isinstance(t, torch.Tensor):
        raise B.ChmError(B.ERR_ARG, name + " must be a tensor")
    shape = t.shape
    if len(shape) != 2:
        raise B.ChmError(B.ERR_ARG, name + " must be a matrix")
    r, c = shape
    if not t.is_cuda or (device is not None and t.get_device() != device):
        raise B.ChmError(B.ERR_ARG, name + " must be on the GPU, the same as the others")
    if dtype is not None and t.dtype != dtype:
        raise B.ChmError(B.ERR_ARG, "%s must be %s" % (name, dtype))
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        raise B.ChmError(B.ERR_ARG, "%s must be %s x %s, is %d x %d" % (name, rows, cols, r, c))
    ld, step = t.stride()
    if c > 1 and step != 1:
        raise B.ChmError(B.ERR_ARG, name + " must have unit stride along its rows")
    if r <= 1:
        return c or 1
    if ld < c:
        raise B.ChmError(B.ERR_ARG, name + "'s rows must not overlap")
    return ld or 1


class _Other:
    """another stream or device than the current one, made current for the launches and allocations within; the caller's tensors are
    not given to anybody else before the work there has been done"""

    def __init__(self, stream, device, tensors):
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=torch.device("cuda", device))
        self.scopes = [torch.cuda.device(device)] + ([torch.cuda.stream(stream)] if stream is not None else [])
        self.device, self.tensors = device, tensors

    def __enter__(self):
        for scope in self.scopes:
            scope.__enter__()
        stream = torch.cuda.current_stream()
        for t in self.tensors:
            if t is not None:
                t.record_stream(stream)
        return torch._C._cuda_getCurrentRawStream(self.device)

    def __exit__(self, *exc):
        for scope in reversed(self.scopes):
            scope.__exit__(*exc)


class _Current:
    """the current stream of the current device: nothing to change"""

    def __init__(self, ptr):
        self.ptr = ptr

    def __enter__(self):
        return self.ptr

    def __exit__(self, *exc):
        pass


def _scope(stream, device, *tensors):
    """scope of a call on the GPU of that index with these tensors: the stream to launch on, current for what is allocated within"""
    if stream is None and torch._C._cuda_getDevice() == device:
        return _Current(torch._C._cuda_getCurrentRawStream(device))
    return _Other(stream, device, tensors)


def _unrecorded(*tensors, kept=False):
    """refuses inputs whose derivatives would be lost; kept: the caller has what the gradient's call wants"""
    if not kept and any([t.requires_grad for t in tensors]) and torch.is_grad_enabled():
        raise B.ChmError(B.ERR_ARG, "the result would carry no gradient to inputs that require one: call under torch.no_grad() and take the "
                                    "gradients from ffn_backward, embedding_gradient, Rotary.gradient and attention_backward")
    if forward_ad._current_level >= 0 and any([forward_ad.unpack_dual(t).tangent is not None for t in tensors]):
        raise B.ChmError(B.ERR_ARG, "the result would carry no tangent: there are no derivatives in forward mode")


def _bytes(n, like):
    return like.new_empty(max(n, 16), dtype=torch.uint8)


def _ffn(x, w_gate, w_up, w_down, activation):
    """the call's description, its sizes, type and GPU"""
    _need(activation in ACTIVATIONS, "activation must be silu, gelu or gelu_tanh")
    ld_x = _matrix("x", x)
    dtype, dev = x.dtype, x.get_device()
    _need(dtype in (torch.bfloat16, torch.float16), "x must be bfloat16 or float16")
    T, D = x.shape
    ld_gate = _matrix("w_gate", w_gate, None, D, dtype, dev)
    F = w_gate.shape[0]
    ld_up = _matrix("w_up", w_up, F, D, dtype, dev)
    ld_down = _matrix("w_down", w_down, D, F, dtype, dev)
    d = B.Ffn(DTYPES[dtype], ACTIVATIONS[activation], T, D, F, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(),
              ld_x, ld_gate, ld_up, ld_down)
    return d, T, D, F, dtype, dev


def ffn_forward(x, w_gate, w_up, w_down, activation="silu", save=False, out=None, stream=None):
    """chm_ffn_forward: y = (act(x w_gate^T) * (x w_up^T)) w_down^T for x [tokens, width], w_gate and w_up [features, width],
    w_down [width, features], all bfloat16 or all float16, rows of any stride.  activation: "silu", "gelu", "gelu_tanh".  With
    save=True returns (y, saved), `saved` being what ffn_backward wants (opaque; 6 bytes per token and feature)."""
    d, T, D, F, dtype, dev = _ffn(x, w_gate, w_up, w_down, activation)
    ld_y = D if out is None else _matrix("out", out, T, D, dtype, dev)
    _unrecorded(x, w_gate, w_up, w_down, kept=save)
    lib = B.lib()
    with _scope(stream, dev, x, w_gate, w_up, w_down, out) as st:
        need, scratch = C.c_uint64(), C.c_uint64()
        B._check(lib.chm_ffn_sizes(d, None, need, scratch, None))
        saved = None
        if save:
            saved = _bytes(need.value, x)
            d.saved = saved.data_ptr()
        if out is None:
            out = x.new_empty((T, D))
        ws = _bytes(scratch.value, x)
        B._check(lib.chm_ffn_forward(d, out.data_ptr(), ld_y, ws.data_ptr(), scratch, st))
    return (out, saved) if save else out


def ffn_backward(dy, x, w_gate, w_up, w_down, saved, activation="silu", grads=None, accumulate=False, out=None, stream=None):
    """chm_ffn_backward: (dx, dw_gate, dw_up, dw_down) for dy, the gradient with respect to ffn_forward's result.  `grads`: the three
    weights' gradients to write, or with accumulate=True to add to; of the weights' type or float32.  `out`: dx to write."""
    d, T, D, F, x_dtype, dev = _ffn(x, w_gate, w_up, w_down, activation)
    ld_dy = _matrix("dy", dy, T, D, x_dtype, dev)
    _need(isinstance(saved, torch.Tensor) and saved.get_device() == dev and saved.dtype == torch.uint8 and saved.is_contiguous(),
          "saved must be what ffn_forward returned")
    ld_dx = D if out is None else _matrix("out", out, T, D, x_dtype, dev)
    if grads is None:
        _need(not accumulate, "accumulate needs grads")
        dtype, lds = x_dtype, (D, D, F)
    else:
        _need(len(grads) == 3 and all(isinstance(t, torch.Tensor) for t in grads), "grads must be three matrices")
        dtype = grads[0].dtype
        _need(dtype in (x_dtype, torch.float32), "grads must be of the weights' type or float32")
        lds = (_matrix("grads[0]", grads[0], F, D, dtype, dev), _matrix("grads[1]", grads[1], F, D, dtype, dev),
               _matrix("grads[2]", grads[2], D, F, dtype, dev))
    _unrecorded(dy, x, w_gate, w_up, w_down, kept=True)
    lib = B.lib()
    with _scope(stream, dev, dy, x, w_gate, w_up, w_down, saved, out, *(grads or ())) as st:
        if out is None:
            out = x.new_empty((T, D))
        if grads is None:
            grads = (x.new_empty((F, D)), x.new_empty((F, D)), x.new_empty((D, F)))
        d.saved = saved.data_ptr()
        g = B.FfnGradients(dy.data_ptr(), out.data_ptr(), grads[0].data_ptr(), grads[1].data_ptr(), grads[2].data_ptr(),
                           ld_dy, ld_dx, *lds, DTYPES[dtype], 1 if accumulate else 0)
        need, scratch = C.c_uint64(), C.c_uint64()
        B._check(lib.chm_ffn_sizes(d, g, need, None, scratch))
        _need(saved.numel() >= need.value, "saved is not of a forward call of these sizes")
        ws = _bytes(scratch.value, x)
        B._check(lib.chm_ffn_backward(d, g, ws.data_ptr(), scratch, st))
    return (out,) + tuple(grads)


def _tokens(tokens, device):
    """checks the tokens and returns their bits and number"""
    _need(isinstance(tokens, torch.Tensor) and tokens.is_cuda and tokens.get_device() == device, "tokens must be on the same GPU as the others")
    _need(tokens.dtype in INDEX_BITS, "tokens must be int32 or int64")
    _need(tokens.is_contiguous(), "tokens must be contiguous")
    return INDEX_BITS[tokens.dtype], tokens.numel()


def embedding_lookup(tokens, table, scale=1.0, out=None, stream=None):
    """chm_embedding_lookup: rows scale * table[token], [tokens.numel(), width]; zeros for a token outside the table (padding,
    or a token of another shard)."""
    ld = _matrix("table", table)
    dtype, dev = table.dtype, table.get_device()
    _need(dtype in DTYPES, "table must be float32, bfloat16 or float16")
    bits, n = _tokens(tokens, dev)
    rows, width = table.shape
    ld_out = width if out is None else _matrix("out", out, n, width, dtype, dev)
    _unrecorded(table)
    with _scope(stream, dev, tokens, table, out) as st:
        if out is None:
            out = table.new_empty((n, width))
        B._check(B.lib().chm_embedding_lookup(DTYPES[dtype], bits, tokens.data_ptr(), n, table.data_ptr(), ld, rows, width, scale,
                                              out.data_ptr(), ld_out, st))
    return out


def embedding_gradient(dy, tokens, rows=None, scale=1.0, out=None, accumulate=False, stream=None):
    """chm_embedding_gradient: the table's gradient [rows, width], row v being scale times the sum of dy's rows at the places of
    token v.  `out`: the gradient to write, or with accumulate=True to add to (rows without a token are not touched); of dy's type
    or float32."""
    ld = _matrix("dy", dy)
    dtype, dev = dy.dtype, dy.get_device()
    _need(dtype in DTYPES, "dy must be float32, bfloat16 or float16")
    bits, n = _tokens(tokens, dev)
    _need(dy.shape[0] == n, "dy must have a row for each token")
    width = dy.shape[1]
    if out is None:
        _need(rows is not None and rows >= 0 and not accumulate, "rows or, with accumulate, out must be given")
        grad_dtype, ld_out = dtype, width
    else:
        ld_out = _matrix("out", out, rows, width, None, dev)
        rows, grad_dtype = out.shape[0], out.dtype
        _need(grad_dtype in (dtype, torch.float32), "out must be of dy's type or float32")
    _unrecorded(dy, kept=True)
    lib = B.lib()
    with _scope(stream, dev, dy, tokens, out) as st:
        if out is None:
            out = dy.new_empty((rows, width))
        scratch = C.c_uint64()
        B._check(lib.chm_embedding_gradient_scratch(n, rows, width, scratch))
        ws = _bytes(scratch.value, dy)
        B._check(lib.chm_embedding_gradient(DTYPES[dtype], DTYPES[grad_dtype], bits, tokens.data_ptr(), n, dy.data_ptr(), ld, rows, width,
                                            scale, out.data_ptr(), ld_out, 1 if accumulate else 0, ws.data_ptr(), scratch, st))
    return out


PAIRINGS = {"halves": 0, "neighbours": 1}


def _strided(name, t, shape, dtype, device):
    """checks a tensor of that shape (a number: of so many dimensions), whose last dimension has unit stride, and returns its shape"""
    if not isinstance(t, torch.Tensor):
        raise B.ChmError(B.ERR_ARG, name + " must be a tensor")
    got = t.shape
    if (len(got) if type(shape) is int else got) != shape:
        raise B.ChmError(B.ERR_ARG, "%s must be %s, is %s" % (name, "of %d dimensions" % shape if type(shape) is int else list(shape), list(got)))
    if not t.is_cuda or (device is not None and t.get_device() != device):
        raise B.ChmError(B.ERR_ARG, name + " must be on the GPU, the same as the others")
    if dtype is not None and t.dtype != dtype:
        raise B.ChmError(B.ERR_ARG, "%s must be %s" % (name, dtype))
    if got[-1] > 1 and t.stride(-1) != 1:
        raise B.ChmError(B.ERR_ARG, name + " must have unit stride along its last dimension")
    return got


class Rotary:
    """Rotary positions of one or several axes: the description of chm_rotary_turn, made once for a model.

    `sections`: how many pairs each axis turns, one axis behind the other ([64] for text; [16, 24, 24] for time, height and width), or `axes`:
    the axis of every pair, in any order.  Neither: all pairs by one axis.  `frequencies`: radians a position of every pair; without them
    base ** (-i / pairs) for pair i.  `pairing`: "halves" (elements i and i + pairs of a head) or "neighbours" (2 i and 2 i + 1).  Elements behind
    the pairs are copied."""

    def __init__(self, head_dim, sections=None, axes=None, frequencies=None, base=10000.0, pairing="halves"):
        _need(isinstance(head_dim, int) and 2 <= head_dim <= 1 << 20, "head_dim must be a whole number from 2 to 2^20")
        _need(pairing in PAIRINGS, "pairing must be halves or neighbours")
        _need(sections is None or axes is None, "sections or axes, not both")
        if sections is not None:
            sections = list(sections)
            _need(sections and all(isinstance(n, int) and n >= 0 for n in sections), "sections must be whole numbers")
            axes = [a for a, n in enumerate(sections) for _ in range(n)]
        elif axes is None:
            axes = [0] * (len(list(frequencies)) if frequencies is not None else head_dim // 2)
        axes = list(axes)
        _need(all(isinstance(a, int) and 0 <= a < 256 for a in axes), "axes must be whole numbers from 0 to 255")
        pairs = len(axes)
        _need(1 <= pairs <= 128 and 2 * pairs <= head_dim, "there must be 1 to 128 pairs, twice as many elements of a head at least")
        if frequencies is None:
            base = float(base)
            _need(base > 0 and math.isfinite(base), "base must be positive")
            frequencies = [base ** (-i / pairs) for i in range(pairs)]
        frequencies = [float(f) for f in frequencies]
        _need(len(frequencies) == pairs and all(math.isfinite(f) for f in frequencies), "frequencies must be a finite number for each pair")
        self.head_dim, self.pairs, self.axes = head_dim, pairs, len(sections) if sections is not None else max(axes) + 1
        self._frequencies, self._axis = (C.c_double * pairs)(*frequencies), (C.c_int32 * pairs)(*axes)
        self._pairing = PAIRINGS[pairing]

    def _turn(self, name, x, positions, backwards, out, stream):
        n, heads, dim = _strided(name, x, 3, None, None)
        dtype, dev = x.dtype, x.get_device()
        _need(dim == self.head_dim, name + "'s heads must have the elements that were described")
        _need(dtype in DTYPES, name + " must be float32, bfloat16 or float16")
        _need(isinstance(positions, torch.Tensor) and positions.is_cuda and positions.get_device() == dev, "positions must be on the same GPU as the others")
        _need(positions.dtype in INDEX_BITS, "positions must be int32 or int64")
        if positions.dim() == 1 and self.axes == 1:
            positions = positions[None]
        if positions.shape != (self.axes, n):
            raise B.ChmError(B.ERR_ARG, "positions must be %d x %d (axes x tokens)" % (self.axes, n))
        if out is not None:
            _strided("out", out, (n, heads, self.head_dim), dtype, dev)
        _unrecorded(x)
        with _scope(stream, dev, x, positions, out) as st:
            if out is None:
                out = x.new_empty((n, heads, self.head_dim))
            d = B.RotaryTurn(DTYPES[dtype], INDEX_BITS[positions.dtype], self._pairing, self.axes, n, heads, self.head_dim, self.pairs, x.data_ptr(),
                             out.data_ptr(), x.stride(0), x.stride(1), out.stride(0), out.stride(1), positions.data_ptr(), positions.stride(0),
                             positions.stride(1), C.addressof(self._frequencies), C.addressof(self._axis))
            B._check(B.lib().chm_rotary_turn(d, backwards, st))
        return out

    def rotate(self, x, positions, out=None, stream=None):
        """x [tokens, heads, head_dim] (queries, keys, or both side by side; any strides) turned by positions [axes, tokens] (or [tokens] for one
        axis), whole numbers of either sign.  `out` may be x."""
        return self._turn("x", x, positions, 0, out, stream)

    def gradient(self, dy, positions, out=None, stream=None):
        """the gradient of x for dy, that of rotate's result.  `out` may be dy."""
        return self._turn("dy", dy, positions, 1, out, stream)


def _strides(t):
    return t.stride()[:3]


def _attention(q, k, v, scale, cap, slopes, causal, documents, prefix):
    """the call's description, its GPU, and the tensors it points to"""
    batch, tokens, heads, dim = _strided("q", q, 4, None, None)
    dtype, dev = q.dtype, q.get_device()
    _need(dtype is torch.bfloat16 or dtype is torch.float16, "q must be bfloat16 or float16")
    shape = _strided("k", k, 4, dtype, dev)
    keys, kv_heads = shape[1], shape[2]
    _need(shape[0] == batch and shape[3] == dim, "q and k must have the same batch and elements of a head")
    _strided("v", v, shape, dtype, dev)
    _need(kv_heads > 0 and heads > 0 and heads % kv_heads == 0, "the heads of q must be a multiple of those of k and v")
    _need(1 <= dim <= 128, "heads must have 1 to 128 elements")
    scale = dim ** -0.5 if scale is None else float(scale)
    cap = float(cap)
    _need(0 < scale <= 1e30, "scale must be positive, up to 1e30")
    _need(cap >= 0 and math.isfinite(cap) and scale <= 1e30 * (cap or 1.0), "cap must be positive (0: none), scale / cap up to 1e30")
    d = B.Attention(DTYPES[dtype], 1 if causal else 0, batch, tokens, keys, heads, kv_heads, dim, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                    _strides(q), _strides(k), _strides(v), scale, cap)
    held = [q, k, v]
    if slopes is not None:
        _need(isinstance(slopes, torch.Tensor) and slopes.is_cuda and slopes.get_device() == dev and slopes.dtype == torch.float32 and
              tuple(slopes.shape) == (heads,) and slopes.is_contiguous(), "slopes must be a float32 for each head, on the same GPU")
        _need(not slopes.requires_grad, "slopes are constants: they get no gradient")
        d.slopes = slopes.data_ptr()
        held.append(slopes)
    if documents is not None:
        pair = tuple(documents) if isinstance(documents, (tuple, list)) else (documents, documents)
        _need(len(pair) == 2, "documents must be one tensor, or one for the queries and one for the keys")
        for name, t, n in (("q", pair[0], tokens), ("k", pair[1], keys)):
            _strided(name + "'s documents", t, (batch, n), None, dev)
            _need(t.dtype in INDEX_BITS and t.dtype == pair[0].dtype, "documents must be int32 or int64")
        d.index_bits = INDEX_BITS[pair[0].dtype]
        d.q_documents, d.k_documents = pair[0].data_ptr(), pair[1].data_ptr()
        d.ld_q_documents, d.ld_k_documents = pair[0].stride(0), pair[1].stride(0)
        held += pair
    if prefix is not None:
        _need(causal, "a prefix is what a causal mask leaves visible: it needs causal")
        _strided("prefix", prefix, (batch, keys), None, dev)
        _need(prefix.dtype in (torch.bool, torch.uint8), "prefix must be bool or uint8")
        d.prefix, d.ld_prefix = prefix.data_ptr(), prefix.stride(0)
        held.append(prefix)
    return d, dev, held


def attention_forward(q, k, v, scale=None, cap=0.0, slopes=None, causal=True, documents=None, prefix=None, save=False, out=None, stream=None):
    """chm_attention_forward: y [batch, tokens, heads, dim] for q of that shape and k, v [batch, keys, kv_heads, dim], all bfloat16 or all float16, any
    strides; query head h reads key head h // (heads // kv_heads).  Scores are scale q.k (scale: dim ** -0.5), capped to
    cap tanh(. / cap) where cap > 0, less slopes[head] times the distance (slopes: float32 [heads]).

    Query i stands at position i + keys - tokens.  It sees the keys of its document (documents: whole numbers [batch, tokens], or a pair of them for
    queries and keys; outside [0, 2^31 - 1) they stand for none) and, if causal, those up to its own position and those that prefix
    (bool [batch, keys]) names.  One that sees nothing gets zeros.  With save=True returns (y, saved), `saved` being what attention_backward wants
    (opaque; 2 bytes per element of y, 4 per row, with documents or a prefix some 5 per token and key)."""
    d, dev, held = _attention(q, k, v, scale, cap, slopes, causal, documents, prefix)
    if out is not None:
        _strided("out", out, q.shape, q.dtype, dev)
    _unrecorded(q, k, v, kept=save)
    lib = B.lib()
    with _scope(stream, dev, out, *held) as st:
        need, scratch = C.c_uint64(), C.c_uint64()
        B._check(lib.chm_attention_sizes(d, None, need, scratch, None))
        saved = None
        if save:
            saved = _bytes(need.value, q)
            d.saved = saved.data_ptr()
        if out is None:
            out = q.new_empty(q.shape)
        ws = _bytes(scratch.value, q) if scratch.value else None
        B._check(lib.chm_attention_forward(d, out.data_ptr(), B.Strides(*_strides(out)), ws.data_ptr() if ws is not None else None, scratch, st))
    return (out, saved) if save else out


def attention_backward(dy, q, k, v, y, saved, scale=None, cap=0.0, slopes=None, causal=True, documents=None, prefix=None, out=None, stream=None):
    """chm_attention_backward: (dq, dk, dv) for dy, the gradient with respect to y, from attention_forward's y and saved; the other arguments as there
    (documents and prefix by any tensors that hold the same: what they are lies in saved).
    `out`: the three tensors to write (of any strides: the parts of one projection's gradient)."""
    d, dev, held = _attention(q, k, v, scale, cap, slopes, causal, documents, prefix)
    _strided("dy", dy, q.shape, q.dtype, dev)
    _strided("y", y, q.shape, q.dtype, dev)
    _need(isinstance(saved, torch.Tensor) and saved.get_device() == dev and saved.dtype == torch.uint8 and saved.is_contiguous(),
          "saved must be what attention_forward returned")
    if out is not None:
        out = tuple(out)
        _need(len(out) == 3, "out must be three tensors")
        for name, t, like in zip(("out[0]", "out[1]", "out[2]"), out, (q, k, v)):
            _strided(name, t, like.shape, q.dtype, dev)
    _unrecorded(dy)
    _unrecorded(q, k, v, y, kept=True)
    lib = B.lib()
    with _scope(stream, dev, dy, y, saved, *held, *(out or ())) as st:
        if out is None:
            out = (q.new_empty(q.shape), k.new_empty(k.shape), v.new_empty(v.shape))
        d.saved = saved.data_ptr()
        g = B.AttentionGradients(dy.data_ptr(), y.data_ptr(), *[t.data_ptr() for t in out], _strides(dy), _strides(y), *[_strides(t) for t in out])
        need, scratch = C.c_uint64(), C.c_uint64()
        B._check(lib.chm_attention_sizes(d, g, need, None, scratch))
        _need(saved.numel() >= need.value, "saved is not of a forward call of these sizes")
        ws = _bytes(scratch.value, q)
        B._check(lib.chm_attention_backward(d, g, ws.data_ptr(), ws.numel(), st))
    return out


def _dense(t):
    """whether the tensor's elements fill one stretch of memory, in whatever order"""
    n = 1
    for stride, size in sorted((s, k) for s, k in zip(t.stride(), t.shape) if k > 1):
        if stride != n:
            return False
        n *= size
    return True


class Gradients:
    """chm_load_gradients ... chm_free_gradients: the gradients of a stage, whose buffers stay where they are from step to step (where they
    are made anew, as by zero_grad(set_to_none=True), the list is too, which waits for the device).

    `grads`: dense tensors (float32, bfloat16, float16, mixed) on one GPU.  `out`: tensors of the same types, shapes and strides that
    receive the clipped gradients; without it they are clipped in place.  The tensors' memory is kept.  Calls share the handle's workspace:
    one on another stream than the last waits for that one on the GPU (a stream that was handed in lives until then).  A captured call is
    ordered by whoever replays it."""

    def __init__(self, grads, out=None):
        grads = list(grads)
        out = None if out is None else list(out)
        _need(out is None or len(out) == len(grads), "out must have a tensor for each gradient")
        _need(all(isinstance(t, torch.Tensor) for t in grads), "gradients must be tensors")
        _unrecorded(*grads, kept=True)
        self.device = grads[0].device if grads else torch.device("cuda", torch.cuda.current_device())
        items = (B.Gradient * max(len(grads), 1))()
        for i, t in enumerate(grads):
            _need(t.is_cuda and t.device == self.device, "gradients must be on one GPU")
            _need(t.dtype in DTYPES, "gradients must be float32, bfloat16 or float16")
            _need(_dense(t), "gradients must be dense")
            items[i].grad, items[i].n, items[i].dtype = t.data_ptr(), t.numel(), DTYPES[t.dtype]
            if out is not None:
                o = out[i]
                _need(isinstance(o, torch.Tensor) and o.device == t.device and o.dtype == t.dtype and o.shape == t.shape and
                      (t.numel() <= 1 or o.stride() == t.stride() or (o.is_contiguous() and t.is_contiguous())),
                      "out must match the gradients")
                items[i].out = o.data_ptr()
        self._h = C.c_void_p()
        self._tensors = [t.detach() for t in grads + (out or [])]          # aliases: a tensor may be given other memory
        self._last = None                                                  # the stream of the last call
        with torch.cuda.device(self.device):
            B._check(B.lib().chm_load_gradients(items, len(grads), C.byref(self._h)))

    def close(self):
        if getattr(self, "_h", None):
            B.lib().chm_free_gradients(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _ordered(self, st):
        """the current stream (st) goes on behind the handle's last call"""
        if (self._last is None or self._last.cuda_stream != st) and not torch.cuda.is_current_stream_capturing():
            here = torch.cuda.current_stream()
            if self._last is not None:
                here.wait_stream(self._last)
            self._last = here

    def sumsq(self, stream=None):
        """chm_gradient_sumsq: the sum of squares, a float64 tensor of one element on the GPU; those of the stages of a pipeline add up"""
        with _scope(stream, self.device.index) as st:
            self._ordered(st)
            total = torch.empty(1, dtype=torch.float64, device=self.device)
            B._check(B.lib().chm_gradient_sumsq(self._h, total.data_ptr(), st))
        return total

    def clip(self, max_norm, sumsq=None, stream=None):
        """chm_clip_gradients: clips to max_norm and returns the norm, a float32 scalar on the GPU.  `sumsq`: the sum of squares
        over all stages (float64, one element, on the GPU) in place of that of these gradients."""
        max_norm = float(max_norm)
        _need(not math.isnan(max_norm) and max_norm >= 0, "max_norm must not be negative")
        if sumsq is not None:
            _need(isinstance(sumsq, torch.Tensor) and sumsq.device == self.device and sumsq.dtype == torch.float64 and sumsq.numel() == 1,
                  "sumsq must be a float64 tensor of one element")
        with _scope(stream, self.device.index, sumsq) as st:
            self._ordered(st)
            norm = torch.empty((), dtype=torch.float32, device=self.device)
            B._check(B.lib().chm_clip_gradients(self._h, max_norm, None if sumsq is None else sumsq.data_ptr(), norm.data_ptr(), st))
        return norm
