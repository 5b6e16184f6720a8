"""Rotary positions on the GPU against the formula in 64 bits.

Tolerances.  The angle is worked out in 64 bits and reduced to a turn: off by 2^-52 of the turns, and by 2^-25 turns once it is rounded to
float32; sine and cosine are right to 2 units of 2^-24.  A turned element is the sum of two products, so it is off by at most
(|a| + |b|) (2 pi 2^-25 + 4 2^-24 + turns 2^-51) and the rounding of the result to its type.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_21613_amd import binding, operators
    binding.lib()
    return operators


def heads(seed, n, H, d, dtype, pad=0, shift=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    buf = torch.full((n * (H * d + pad) + shift,), float("nan"), dtype=dtype, device="cuda")
    t = buf[shift:].view(n, H * d + pad)[:, :H * d].unflatten(1, (H, d))
    t.copy_(torch.randn((n, H, d), generator=g, device="cuda"))
    return t


def formula(x, positions, axes, frequencies, pairing, sign):
    """(value, bound of the error before rounding)"""
    P = len(axes)
    f = torch.tensor(frequencies, dtype=torch.float64, device="cuda")
    angle = positions.double()[torch.tensor(axes, device="cuda")].T * f
    c, s = torch.cos(angle)[:, None], sign * torch.sin(angle)[:, None]
    e = (2 * math.pi * 2.0 ** -25 + 4 * 2.0 ** -24 + angle.abs() * 2.0 ** -51)[:, None]
    x = x.double()
    out, off = x.clone(), torch.zeros_like(x)
    first, second = (slice(0, P), slice(P, 2 * P)) if pairing == "halves" else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    a, b = x[..., first], x[..., second]
    out[..., first], out[..., second] = a * c - b * s, a * s + b * c
    off[..., first] = off[..., second] = (a.abs() + b.abs()) * e
    return out, off


def check(got, want, off):
    err = (got.double() - want).abs()
    tol = off + torch.clamp((want.abs() + off) * U[got.dtype], min=TINY[got.dtype])
    assert bool((err <= tol * 1.0001).all()), (float((err - tol).max()), [int(i) for i in (err > tol).nonzero()[0]])


def frequencies_of(P, base=10000.0):
    return [base ** (-i / P) for i in range(P)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
@pytest.mark.parametrize("n,H,d,sections", [(1, 1, 2, [1]), (1, 40, 128, [64]), (2, 3, 8, [4]), (7, 5, 82, [18, 19]), (300, 12, 128, [16, 24, 24]), (33, 2, 256, [128]),
                                            (65, 7, 80, [40]), (1000, 1, 64, [3, 9]), (5, 100, 96, [0, 5, 17, 1]), (129, 9, 37, [11]), (3, 2, 5000, [100])])
def test_turn_and_back(ops, n, H, d, sections, pairing, dtype):
    P = sum(sections)
    axes = [a for a, k in enumerate(sections) for _ in range(k)]
    g = torch.Generator().manual_seed(n)
    pos = torch.randint(-50, 5000, (len(sections), n), generator=g).cuda()
    rope = ops.Rotary(d, sections, pairing=pairing)
    x = heads(n, n, H, d, dtype)
    for sign, call in ((1, rope.rotate), (-1, rope.gradient)):
        want, off = formula(x, pos, axes, frequencies_of(P), pairing, sign)
        got = call(x, pos)
        assert got.dtype == dtype and got.is_contiguous()
        check(got, want, off)
        assert torch.equal(call(x, pos.int()), got)
        inplace = x.clone()
        assert call(inplace, pos, out=inplace) is inplace and torch.equal(inplace, got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (5, 7), (8, 0), (64, 8)])
def test_strides_and_alignment(ops, pad, shift, pairing, dtype):
    n, H, d = 50, 6, 72
    x, out = heads(1, n, H, d, dtype, pad, shift), heads(2, n, H, d, dtype, pad + 2, shift + 1)
    rope = ops.Rotary(d, [10, 20], pairing=pairing)
    pos = torch.arange(3 * n, device="cuda").view(3, n)[::2]
    want, off = formula(x, pos, [0] * 10 + [1] * 20, frequencies_of(30), pairing, 1)
    assert rope.rotate(x, pos, out=out) is out
    check(out, want, off)
    assert bool(torch.isnan(out._base[:shift + 1]).all()) and bool(torch.isnan(out._base[shift + 1:].view(n, -1)[:, H * d:]).all())
    part = rope.rotate(x[:, 1:4], pos, out=x[:, 1:4])           # the middle heads in place, the others left alone
    check(part, want[:, 1:4], off[:, 1:4])
    assert torch.equal(x[:, :1], heads(1, n, H, d, dtype, pad, shift)[:, :1]) and bool(torch.isfinite(x[:, 4:]).all())
    by_head = heads(1, H, n, d, dtype).transpose(0, 1)
    want, off = formula(by_head, pos, [0] * 10 + [1] * 20, frequencies_of(30), pairing, 1)
    check(rope.rotate(by_head, pos), want, off)


def test_axes_and_frequencies_of_any_kind(ops):
    n, H, d = 70, 3, 64
    axes, freq = [0, 2, 1, 0, 2, 1, 2, 2, 0] * 3, [0.01 * i - 0.1 for i in range(27)]
    x = heads(4, n, H, d, torch.float32)
    pos = torch.randint(-1000, 1000, (3, n), device="cuda")
    for pairing in ("halves", "neighbours"):
        want, off = formula(x, pos, axes, freq, pairing, 1)
        check(ops.Rotary(d, axes=axes, frequencies=freq, pairing=pairing).rotate(x, pos), want, off)
    one = ops.Rotary(d)                                          # all pairs by one axis: positions may be a vector
    want, off = formula(x, pos[:1], [0] * 32, frequencies_of(32), "halves", 1)
    check(one.rotate(x, pos[0]), want, off)
    shared = pos[0, :1].expand(n)                                # one position for all tokens
    want, off = formula(x, shared[None], [0] * 32, frequencies_of(32), "halves", 1)
    check(one.rotate(x, shared), want, off)


@pytest.mark.parametrize("start", [1 << 20, (1 << 31) - 40, 1 << 40])
def test_far_positions(ops, start):
    n = 40
    pos = (torch.arange(n, device="cuda") + start)[None]
    x = heads(5, n, 2, 64, torch.float32)
    want, off = formula(x, pos, [0] * 32, frequencies_of(32), "halves", 1)
    check(ops.Rotary(64).rotate(x, pos), want, off)
    if start < 1 << 31:
        assert torch.equal(ops.Rotary(64).rotate(x, pos.int()), ops.Rotary(64).rotate(x, pos))


def test_gradient_is_the_transpose(ops):
    """<dy, rotate(x)> = <gradient(dy), x>, and differences of the formula along a direction"""
    rope = ops.Rotary(96, [10, 12, 20], pairing="neighbours")
    n = 64
    pos = torch.randint(0, 900, (3, n), device="cuda")
    x, dy = heads(1, n, 4, 96, torch.float32), heads(2, n, 4, 96, torch.float32)
    a = (dy.double() * rope.rotate(x, pos).double()).sum()
    b = (rope.gradient(dy, pos).double() * x.double()).sum()
    size = (dy.double().abs() * x.double().abs()).sum() * 2
    assert abs(float(a - b)) <= float(size) * 2 * (2 * math.pi * 2.0 ** -25 + 5 * 2.0 ** -24)
    along, step = heads(3, n, 4, 96, torch.float32).double(), 1e-3
    axes = [0] * 10 + [1] * 12 + [2] * 20
    up, down = (formula(x.double() + s * step * along, pos, axes, frequencies_of(42), "neighbours", 1)[0] for s in (1, -1))
    slope = float((dy.double() * (up - down)).sum()) / (2 * step)
    here = float((rope.gradient(dy, pos).double() * along).sum())
    assert abs(slope - here) <= 2 * float((dy.double().abs() * along.abs()).sum()) * (2 * math.pi * 2.0 ** -25 + 5 * 2.0 ** -24) + 1e-9


def test_many_tokens(ops):
    """offsets beyond 32 bits"""
    n, H, d = 140000, 128, 128
    x = torch.empty((n, H, d), dtype=torch.bfloat16, device="cuda").normal_()
    pos = torch.arange(n, device="cuda")
    rope = ops.Rotary(d)
    y = rope.rotate(x, pos)
    for s in (slice(0, 64), slice(n - 64, n)):
        want, off = formula(x[s], pos[None, s], [0] * 64, frequencies_of(64), "halves", 1)
        check(y[s], want, off)
    assert ops.Rotary(d).rotate(x[:0], pos[:0]).shape == (0, H, d) and rope.rotate(x[:5, :0], pos[:5]).shape == (5, 0, d)


def test_refusals(ops):
    from paper_2508_21613_amd.binding import ChmError
    rope = ops.Rotary(64, [8, 24])
    x, pos = heads(1, 20, 4, 64, torch.bfloat16), torch.zeros((2, 20), dtype=torch.int64, device="cuda")
    for args, kw in (((x.cpu(), pos), {}), ((x, pos.cpu()), {}), ((x[..., :32], pos), {}), ((x[0], pos), {}), ((x, pos[0]), {}), ((x, pos[:, :7]), {}), ((x, pos.float()), {}),
                     ((x.double(), pos), {}), ((x.transpose(1, 2), pos), {}), ((x, pos), dict(out=x[:, :2])), ((x, pos), dict(out=x.half())), ((None, pos), {}), ((x, None), {}),
                     ((x[:, 1:], pos), dict(out=x[:, :3])), ((x, pos), dict(out=x[:1].expand(20, -1, -1)))):
        with pytest.raises(ChmError):
            rope.rotate(*args, **kw)
    x = x.clone().requires_grad_(True)
    with pytest.raises(ChmError):
        rope.rotate(x, pos)
    with torch.no_grad():
        assert rope.rotate(x, pos).shape == x.shape


def test_captured_and_on_another_stream(ops):
    rope = ops.Rotary(64, [8, 24])
    x, pos = heads(1, 200, 8, 64, torch.bfloat16), torch.randint(0, 99, (2, 200), device="cuda")
    want = rope.rotate(x, pos)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    got = rope.rotate(x, pos, stream=stream)
    stream.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = rope.rotate(x, pos)
    for i in range(4):
        x.add_(1)
        pos.add_(i)
        graph.replay()
        want = rope.rotate(x, pos)
        torch.cuda.synchronize()
        assert torch.equal(y, want)
