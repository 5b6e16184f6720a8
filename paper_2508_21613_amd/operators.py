"""Operators of a pipeline stage's training step, over torch tensors: the calls of include/chm_operators.h.

The gated feed-forward block forward and backward, the embedding's lookup and gradient, the global gradient norm with clipping.
As everywhere in this package torch provides device memory and streams; every value is computed by the library's HIP kernels, and
without a usable GPU the calls fail.  A call works on the current stream, or on `stream`; scratch and results that the caller does
not hand in are allocated on that stream.  Inputs must be ready there, as with any torch call.  Results must not lie over inputs or each
other (ffn_forward's may lie over x).  Wrong arguments raise binding.ChmError with the library's code.

Results are no part of autograd's graph; the gradients are calls of their own.  While torch records gradients, inputs that require one are
taken only where the caller asks for what the gradient's call wants (ffn_forward with save=True): anything else would lose it without a word.
"""
import ctypes as C
import math

import torch

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


def _unrecorded(*tensors):
    if any([t.requires_grad for t in tensors]) and torch.is_grad_enabled():
        raise B.ChmError(B.ERR_ARG, "the result would carry no gradient to inputs that require one: call under torch.no_grad() and take the "
                                    "gradients from ffn_backward and embedding_gradient")


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
    if not save:
        _unrecorded(x, w_gate, w_up, w_down)
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
