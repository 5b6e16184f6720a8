"""The operators of a pipeline stage's training step, over torch tensors: the calls of include/chm_operators.h.

The gated feed-forward block forward and backward, the embedding's lookup and gradient, the global gradient norm with clipping.
As everywhere in this package torch provides device memory and streams; every value is computed by the library's HIP kernels, and
without a usable GPU the calls fail.  A call works on the current stream, or on `stream`; scratch and results that the caller does
not hand in are allocated on that stream.  Inputs used there must be ready there, as with any torch call.  Wrong arguments raise
binding.ChmError with the library's code.
"""
import ctypes as C
import math

import torch

from . import binding as B

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}


def _need(ok, what):
    if not ok:
        raise B.ChmError(B.ERR_ARG, what)


def _matrix(name, t, rows=None, cols=None, dtype=None, device=None):
    """checks a row-major matrix (unit stride along rows) and returns the elements from one row to the next"""
    _need(isinstance(t, torch.Tensor) and t.dim() == 2, name + " must be a matrix")
    _need(t.is_cuda, name + " must be on the GPU")
    _need(device is None or t.device == device, name + " must be on the same GPU as the others")
    _need(dtype is None or t.dtype == dtype, "%s must be %s" % (name, dtype))
    _need((rows is None or t.shape[0] == rows) and (cols is None or t.shape[1] == cols),
          "%s must be %s x %s, is %s" % (name, rows, cols, tuple(t.shape)))
    _need(t.shape[1] <= 1 or t.stride(1) == 1, name + " must have unit stride along its rows")
    if t.shape[0] <= 1:
        return max(t.shape[1], 1)
    _need(t.stride(0) >= t.shape[1], name + "'s rows must not overlap")
    return max(t.stride(0), 1)


class _Stream:
    """the stream of a call, made current for the allocations within"""

    def __init__(self, stream, device):
        current = torch.cuda.current_stream(device)
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=device)
        self.other = stream is not None and stream != current
        self.device = device
        self.scope = torch.cuda.stream(stream) if self.other else None
        self.ptr = C.c_void_p((stream if self.other else current).cuda_stream)

    def __enter__(self):
        self.guard = None
        if torch.cuda.current_device() != self.device.index:
            self.guard = torch.cuda.device(self.device)
            self.guard.__enter__()
        if self.scope is not None:
            self.scope.__enter__()
        return self.ptr

    def __exit__(self, *exc):
        if self.scope is not None:
            self.scope.__exit__(*exc)
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _bytes(n, device):
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device=device)


def _ffn(x, w_gate, w_up, w_down, activation):
    _need(activation in ACTIVATIONS, "activation must be one of %s" % ", ".join(ACTIVATIONS))
    ld_x = _matrix("x", x)
    _need(x.dtype in (torch.bfloat16, torch.float16), "x must be bfloat16 or float16")
    T, D = x.shape
    d = B.Ffn()
    d.ld_gate = _matrix("w_gate", w_gate, None, D, x.dtype, x.device)
    F = w_gate.shape[0]
    d.ld_up = _matrix("w_up", w_up, F, D, x.dtype, x.device)
    d.ld_down = _matrix("w_down", w_down, D, F, x.dtype, x.device)
    d.ld_x, d.dtype, d.activation = ld_x, DTYPES[x.dtype], ACTIVATIONS[activation]
    d.tokens, d.width, d.features = T, D, F
    d.x, d.w_gate, d.w_up, d.w_down = x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr()
    return d


def ffn_forward(x, w_gate, w_up, w_down, activation="silu", save=False, out=None, stream=None):
    """chm_ffn_forward: y = (act(x w_gate^T) * (x w_up^T)) w_down^T for x [tokens, width], w_gate and w_up [features, width],
    w_down [width, features], all bfloat16 or all float16, rows of any stride.  activation: "silu", "gelu", "gelu_tanh".  With
    save=True returns (y, saved), `saved` being what ffn_backward wants (opaque; 6 bytes per token and feature)."""
    d = _ffn(x, w_gate, w_up, w_down, activation)
    if out is not None:
        ld_y = _matrix("out", out, d.tokens, d.width, x.dtype, x.device)
    with _Stream(stream, x.device) as st:
        need, scratch = C.c_uint64(), C.c_uint64()
        B._check(B.lib().chm_ffn_sizes(C.byref(d), None, C.byref(need), C.byref(scratch), None))
        saved = _bytes(need.value, x.device) if save else None
        d.saved = saved.data_ptr() if save else None
        if out is None:
            out = torch.empty((d.tokens, d.width), dtype=x.dtype, device=x.device)
            ld_y = d.width
        ws = _bytes(scratch.value, x.device)
        B._check(B.lib().chm_ffn_forward(C.byref(d), out.data_ptr(), ld_y, ws.data_ptr(), ws.numel(), st))
    return (out, saved) if save else out


def ffn_backward(dy, x, w_gate, w_up, w_down, saved, activation="silu", grads=None, accumulate=False, out=None, stream=None):
    """chm_ffn_backward: (dx, dw_gate, dw_up, dw_down) for dy, the gradient with respect to ffn_forward's result.  `grads`: the three
    weights' gradients to write, or with accumulate=True to add to; of the weights' type or float32.  `out`: dx to write."""
    d = _ffn(x, w_gate, w_up, w_down, activation)
    T, D, F, dev = d.tokens, d.width, d.features, x.device
    g = B.FfnGradients()
    g.ld_dy = _matrix("dy", dy, T, D, x.dtype, dev)
    _need(isinstance(saved, torch.Tensor) and saved.is_cuda and saved.device == dev and saved.dtype == torch.uint8, "saved must be what ffn_forward returned")
    if out is not None:
        g.ld_dx = _matrix("out", out, T, D, x.dtype, dev)
    if grads is None:
        _need(not accumulate, "accumulate needs grads")
        dtype = x.dtype
    else:
        _need(len(grads) == 3 and all(isinstance(t, torch.Tensor) for t in grads), "grads must be three matrices")
        dtype = grads[0].dtype
        _need(dtype in (x.dtype, torch.float32), "grads must be of the weights' type or float32")
        g.ld_dw_gate = _matrix("grads[0]", grads[0], F, D, dtype, dev)
        g.ld_dw_up = _matrix("grads[1]", grads[1], F, D, dtype, dev)
        g.ld_dw_down = _matrix("grads[2]", grads[2], D, F, dtype, dev)
    g.grad_dtype, g.accumulate = DTYPES[dtype], int(bool(accumulate))
    with _Stream(stream, dev) as st:
        if out is None:
            out = torch.empty((T, D), dtype=x.dtype, device=dev)
            g.ld_dx = D
        if grads is None:
            grads = [torch.empty((F, D), dtype=dtype, device=dev), torch.empty((F, D), dtype=dtype, device=dev),
                     torch.empty((D, F), dtype=dtype, device=dev)]
            g.ld_dw_gate, g.ld_dw_up, g.ld_dw_down = D, D, F
        d.saved = saved.data_ptr()
        g.dy, g.dx = dy.data_ptr(), out.data_ptr()
        g.dw_gate, g.dw_up, g.dw_down = (t.data_ptr() for t in grads)
        need, scratch = C.c_uint64(), C.c_uint64()
        B._check(B.lib().chm_ffn_sizes(C.byref(d), C.byref(g), C.byref(need), None, C.byref(scratch)))
        _need(saved.numel() >= need.value, "saved is not of a forward call of these sizes")
        ws = _bytes(scratch.value, dev)
        B._check(B.lib().chm_ffn_backward(C.byref(d), C.byref(g), ws.data_ptr(), ws.numel(), st))
    return (out,) + tuple(grads)


def _tokens(tokens, device):
    _need(isinstance(tokens, torch.Tensor) and tokens.is_cuda and tokens.dtype in (torch.int32, torch.int64), "tokens must be int32 or int64 on the GPU")
    _need(device is None or tokens.device == device, "tokens must be on the same GPU as the others")
    _need(tokens.is_contiguous(), "tokens must be contiguous")
    return tokens.element_size() * 8


def embedding_lookup(tokens, table, scale=1.0, out=None, stream=None):
    """chm_embedding_lookup: rows scale * table[token], [tokens.numel(), width]; zeros for a token outside the table (padding,
    or a token of another shard)."""
    ld = _matrix("table", table)
    _need(table.dtype in DTYPES, "table must be float32, bfloat16 or float16")
    bits, n, (rows, width) = _tokens(tokens, table.device), tokens.numel(), table.shape
    if out is not None:
        ld_out = _matrix("out", out, n, width, table.dtype, table.device)
    with _Stream(stream, table.device) as st:
        if out is None:
            out = torch.empty((n, width), dtype=table.dtype, device=table.device)
            ld_out = width
        B._check(B.lib().chm_embedding_lookup(DTYPES[table.dtype], bits, tokens.data_ptr(), n, table.data_ptr(), ld, rows, width, scale,
                                              out.data_ptr(), ld_out, st))
    return out


def embedding_gradient(dy, tokens, rows=None, scale=1.0, out=None, accumulate=False, stream=None):
    """chm_embedding_gradient: the table's gradient [rows, width], row v being scale times the sum of dy's rows at the places of
    token v.  `out`: the gradient to write, or with accumulate=True to add to (rows without a token are not touched); of dy's type
    or float32."""
    ld = _matrix("dy", dy)
    _need(dy.dtype in DTYPES, "dy must be float32, bfloat16 or float16")
    bits, n, width = _tokens(tokens, dy.device), tokens.numel(), dy.shape[1]
    _need(dy.shape[0] == n, "dy must have a row for each token")
    _need(rows is not None or out is not None, "rows or out must be given")
    _need(out is not None or not accumulate, "accumulate needs out")
    if out is not None:
        ld_out = _matrix("out", out, rows, width, None, dy.device)
        rows = out.shape[0]
        _need(out.dtype in (dy.dtype, torch.float32), "out must be of dy's type or float32")
    with _Stream(stream, dy.device) as st:
        if out is None:
            _need(rows >= 0, "rows must not be negative")
            out = torch.empty((rows, width), dtype=dy.dtype, device=dy.device)
            ld_out = width
        scratch = C.c_uint64()
        B._check(B.lib().chm_embedding_gradient_scratch(n, width, C.byref(scratch)))
        ws = _bytes(scratch.value, dy.device)
        B._check(B.lib().chm_embedding_gradient(DTYPES[dy.dtype], DTYPES[out.dtype], bits, tokens.data_ptr(), n, dy.data_ptr(), ld, rows, width,
                                                scale, out.data_ptr(), ld_out, int(bool(accumulate)), ws.data_ptr(), ws.numel(), st))
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
    """chm_load_gradients ... chm_free_gradients: the gradients of a stage, whose buffers stay where they are from step to step.

    `grads`: dense tensors (float32, bfloat16, float16, mixed) on one GPU.  `out`: tensors of the same types, shapes and strides that
    receive the clipped gradients; without it they are clipped in place.  The tensors are kept alive."""

    def __init__(self, grads, out=None):
        grads = list(grads)
        out = None if out is None else list(out)
        _need(out is None or len(out) == len(grads), "out must have a tensor for each gradient")
        self.device = grads[0].device if grads else torch.device("cuda", torch.cuda.current_device())
        items = (B.Gradient * max(len(grads), 1))()
        for i, t in enumerate(grads):
            _need(isinstance(t, torch.Tensor) and t.is_cuda and t.device == self.device, "gradients must be on one GPU")
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
        self._tensors = (grads, out)
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

    def sumsq(self, stream=None):
        """chm_gradient_sumsq: the sum of squares, a float64 tensor of one element on the GPU; those of the stages of a pipeline add up"""
        with _Stream(stream, self.device) as st:
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
        with _Stream(stream, self.device) as st:
            norm = torch.empty((), dtype=torch.float32, device=self.device)
            B._check(B.lib().chm_clip_gradients(self._h, max_norm, None if sumsq is None else sumsq.data_ptr(), norm.data_ptr(), st))
        return norm
