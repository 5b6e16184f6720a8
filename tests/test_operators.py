"""The operators of a training step (feed-forward block, embedding, gradient norm and clipping) on the GPU against their
formulas in 64 bits.

Tolerances.  A value rounded to a type of unit roundoff u is off by at most u |value| (for float16 at least 2^-25); where such
values enter a sum their errors are independent, with a standard deviation of that bound / sqrt(3), and the sum is allowed six
standard deviations of the total, plus its own rounding.  float32 sums of k terms are allowed sqrt(k) roundings of 2^-24 of the
root of the summed squares, six standard deviations again.  A term that is left out, doubled or misplaced is some
ten times larger than that at the sizes used here.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -12, torch.float32: 2.0 ** -25}
U = {k: 2 * v for k, v in U.items()}             # unit roundoff: half a unit in the last place of 1.0
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
ACC = 2.0 ** -24


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


def normal(g, rows, cols, dtype, std=1.0, pad=0, shift=0):
    """rows x cols normal numbers in rows of cols + pad elements, `shift` elements into their buffer"""
    buf = torch.full((rows * (cols + pad) + shift,), float("nan"), dtype=dtype, device="cuda")
    t = buf[shift:].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.randn(rows, cols, generator=g, device="cuda") * std)
    return t


# ------------------------------------------------------------------------------------------------ feed-forward block
def act_of(act, g):
    """the activation, its derivative, and a bound of its second derivative"""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s)), 0.5
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi), 0.8
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g), 1.0


def rounded(v, dtype):
    """variance of the error of rounding v"""
    return (torch.clamp(v.abs() * U[dtype], min=TINY[dtype])) ** 2 / 3


def summed(a, b, k):
    """variance of the float32 roundings of the product a b over k sums"""
    return (ACC ** 2 * k) * ((a * a) @ (b * b))


def formula(x, wg, wu, wd, act, dy=None):
    """{name: (value, variance of the error)} in 64 bits for inputs of 16 bits"""
    dtype = x.dtype
    x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
    T, D = x.shape
    F = wg.shape[0]
    g, u = x @ wg.T, x @ wu.T
    a, da, dda = act_of(act, g)
    vg, vu = summed(x, wg.T, D), summed(x, wu.T, D)
    h = a * u
    vh = rounded(h, dtype) + (da * u) ** 2 * vg + a ** 2 * vu + (8 * ACC * h) ** 2
    out = {"y": (h @ wd.T, vh @ (wd * wd).T + summed(h, wd.T, F))}
    if dy is None:
        return out
    dy = dy.double()
    vg, vu = vg + (2.0 ** -15 * g) ** 2 / 3, vu + (2.0 ** -15 * u) ** 2 / 3     # 24 bits (16 significant) are kept between the passes
    vh = rounded(h, dtype) + (da * u) ** 2 * vg + a ** 2 * vu + (8 * ACC * h) ** 2
    dh = dy @ wd
    vdh = summed(dy, wd, D)
    du, dg = dh * a, dh * u * da
    vdu = a ** 2 * vdh + (dh * da) ** 2 * vg + rounded(du, dtype) + (8 * ACC * du) ** 2
    vdg = (u * da) ** 2 * vdh + (dh * da) ** 2 * vu + (dh * u * dda) ** 2 * vg + rounded(dg, dtype) + (8 * ACC * dh * u) ** 2
    out["dx"] = (dg @ wg + du @ wu, vdg @ (wg * wg) + vdu @ (wu * wu) + summed(dg, wg, 2 * F) + summed(du, wu, 2 * F))
    out["dw_gate"] = (dg.T @ x, vdg.T @ (x * x) + summed(dg.T, x, T))
    out["dw_up"] = (du.T @ x, vdu.T @ (x * x) + summed(du.T, x, T))
    out["dw_down"] = (dy.T @ h, (dy * dy).T @ vh + summed(dy.T, h, T))
    return out


def check(name, got, want, dtype=None):
    value, var = want
    dtype = dtype or got.dtype
    assert got.shape == value.shape, name
    assert bool(torch.isfinite(got).all()), name
    err = (got.double() - value).abs()
    tol = 6 * var.sqrt() + torch.clamp(value.abs() * U[dtype], min=TINY[dtype]) + 1e-30
    bad = err > tol * 1.0001
    assert not bool(bad.any()), (name, int(bad.sum()), float((err / tol).max()), [int(i) for i in bad.nonzero()[0]])


def ffn_inputs(seed, T, D, F, dtype, pad=0, shift=0):
    g = gen(seed)
    return (normal(g, T, D, dtype, 1.0, pad, shift), normal(g, F, D, dtype, D ** -0.5, pad, shift), normal(g, F, D, dtype, D ** -0.5, pad, shift),
            normal(g, D, F, dtype, F ** -0.5, pad, shift), normal(g, T, D, dtype, 0.5, pad, shift))


NAMES = ("dx", "dw_gate", "dw_up", "dw_down")


def ffn_both(ops, inputs, act, **kw):
    x, wg, wu, wd, dy = inputs
    y, saved = ops.ffn_forward(x, wg, wu, wd, activation=act, save=True)
    grads = ops.ffn_backward(dy, x, wg, wu, wd, saved, activation=act, **kw)
    return dict(zip(("y",) + NAMES, (y,) + grads))


FFN_SHAPES = [(1, 1, 1), (1, 64, 128), (2, 7, 5), (3, 130, 9), (15, 64, 72), (16, 72, 200), (17, 65, 130), (31, 8, 8), (32, 256, 24), (33, 128, 64),
              (63, 200, 96), (64, 513, 1031), (65, 64, 64), (65, 1, 9), (66, 9, 1), (128, 1024, 512), (130, 136, 264), (255, 96, 320), (257, 515, 1001),
              (300, 72, 520), (513, 2048, 256)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", FFN_SHAPES)
def test_ffn_forward_and_backward(ops, shape, dtype):
    act = ("silu", "gelu", "gelu_tanh")[sum(shape) % 3]
    inputs = ffn_inputs(sum(shape), *shape, dtype)
    want = formula(*inputs[:4], act, inputs[4])
    got = ffn_both(ops, inputs, act)
    for k, v in want.items():
        check(k, got[k], v)
    alone = ops.ffn_forward(*inputs[:4], activation=act)                   # without keeping anything: the same bits
    assert torch.equal(alone, got["y"])


# up to 8 tokens the sums go in 1, 2 or 4 slices: ends of rows inside each, several steps a wavefront, fewer sums than one load takes
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", [(1, 8, 8), (1, 7, 9), (1, 1000, 2731), (2, 3001, 800), (3, 8200, 40), (4, 515, 4099), (4, 4096, 72), (5, 1027, 515), (6, 40, 8200),
                                   (7, 2051, 260), (8, 256, 128), (8, 1100, 2049), (9, 515, 1027)])
def test_ffn_slices_of_the_sums(ops, shape, dtype):
    inputs = ffn_inputs(sum(shape), *shape, dtype)
    want = formula(*inputs[:4], "silu", inputs[4])
    got = ffn_both(ops, inputs, "silu")
    for k, v in want.items():
        check(k, got[k], v)
    assert torch.equal(ops.ffn_forward(*inputs[:4]), got["y"])


# tiles of 64 x 64: one to many a product, edges inside, split sums, weights that are packed
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", [(25, 1100, 8000), (37, 2048, 5504), (49, 72, 1000), (60, 1001, 2731), (64, 3000, 3200), (100, 520, 1100), (129, 264, 2000), (49, 8, 16)])
def test_ffn_small_tiles(ops, shape, dtype):
    act = ("silu", "gelu", "gelu_tanh")[sum(shape) % 3]
    inputs = ffn_inputs(sum(shape), *shape, dtype)
    want = formula(*inputs[:4], act, inputs[4])
    for k, v in ffn_both(ops, inputs, act).items():
        check(k, v, want[k])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_ffn_split_sums_on_large_tiles(ops, dtype):
    inputs = ffn_inputs(7, 520, 2051, 5500, dtype)
    want = formula(*inputs[:4], "gelu", inputs[4])
    for k, v in ffn_both(ops, inputs, "gelu").items():
        check(k, v, want[k])


# every kernel of the block, each with every activation: all kinds of tile for every product, whole and split sums, all slices, blocks of
# tokens and ends of the kernels for few tokens (tests/test_operators_host.py asks the library that none is missing)
FFN_KERNELS = [(1, 10, 8), (401, 8, 5888), (2268, 129, 6656), (263, 8384, 75), (309, 4483, 1664), (2711, 3328, 789), (5, 10, 8), (9, 8, 12), (22, 8, 8), (33, 9, 10),
               (14, 64, 64), (1, 256, 256), (34, 64, 64), (5, 128, 256), (17, 64, 256), (49, 8, 12), (10, 7512, 8192), (129, 8576, 8798)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("shape", FFN_KERNELS)
def test_ffn_every_kernel(ops, shape, act, dtype):
    inputs = ffn_inputs(sum(shape), *shape, dtype)
    want = formula(*inputs[:4], act, inputs[4])
    for k, v in ffn_both(ops, inputs, act).items():
        check(k, v, want[k])


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("T", [5, 90])
def test_ffn_activations(ops, act, T):
    inputs = ffn_inputs(3, T, 64, 96, torch.float16)
    inputs[0].mul_(4)                                                      # far into both tails of the activation
    want = formula(*inputs[:4], act, inputs[4])
    for k, v in ffn_both(ops, inputs, act).items():
        check(k, v, want[k])


# The activation's left tail by itself: one token whose projections are g in [-6, -3] and u = 1,024, a down projection that hands h on, so that
# every result is one value of the formula, rounded once to its type.  float32 gets that value to 2^-16: the exponents (up to 25) and the
# argument's square (up to 18) are off by some 2^-23 of themselves.
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("T", [1, 70])
def test_ffn_left_tail_of_the_activations(ops, act, T, dtype):
    F = 192
    g = torch.linspace(-6, -3, F, device="cuda").to(dtype)
    x, wg, wu, dy = (torch.zeros(s, dtype=dtype, device="cuda") for s in ((T, F), (F, F), (F, F), (T, F)))
    x[0, 0], wg[:, 0], wu[:, 0], dy[0] = 1, g, 1024, 1024
    wd = torch.eye(F, device="cuda").to(dtype)
    y, saved = ops.ffn_forward(x, wg, wu, wd, activation=act, save=True)
    grads = [torch.empty((F, F), device="cuda") for _ in range(3)]
    ops.ffn_backward(dy, x, wg, wu, wd, saved, activation=act, grads=grads)
    g = g.double()
    if act == "gelu":
        a = g * torch.special.ndtr(g)
        da = torch.special.ndtr(g) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    else:
        z, dz = (g, 1.0) if act == "silu" else (math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3), math.sqrt(8 / math.pi) * (1 + 3 * 0.044715 * g * g))
        s = torch.sigmoid(z)
        a, da = g * s, s + g * s * torch.sigmoid(-z) * dz
    for name, got, want in (("h", y[0], 1024 * a), ("h again", grads[2][0] / 1024, 1024 * a), ("du", grads[1][:, 0], 1024 * a),
                            ("dg", grads[0][:, 0], 1024 * 1024 * da)):
        beyond = want.abs() > torch.finfo(dtype).max                       # infinite in the type, as the formula's value is
        assert torch.equal(got[beyond].double(), want[beyond].sign() * math.inf), name
        err = (got.double() - want).abs()[~beyond]
        tol = (torch.clamp(want.abs() * U[dtype], min=TINY[dtype]) + 2.0 ** -16 * want.abs())[~beyond]
        assert bool((err <= tol).all()), (name, float((err / tol).max()))


@pytest.mark.parametrize("T", [3, 70, 140])
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (5, 7), (8, 0), (64, 8)])
def test_ffn_strides_and_alignment(ops, T, pad, shift):
    inputs = ffn_inputs(11, T, 72, 104, torch.float16, pad, shift)
    want = formula(*inputs[:4], "silu", inputs[4])
    for k, v in ffn_both(ops, inputs, "silu").items():
        check(k, v, want[k])
    # weights of different strides, results into strided places that start anywhere
    x, wg, wu, wd, dy = inputs
    wu2 = normal(gen(1), 104, 72, torch.float16, 1.0, 16)
    wu2.copy_(wu)
    outs = [normal(gen(2), r, c, torch.float16, 1.0, 5, 3) for r, c in ((T, 72), (T, 72), (104, 72), (104, 72), (72, 104))]
    y, saved = ops.ffn_forward(x, wg, wu2, wd, save=True, out=outs[0])
    assert y is outs[0]
    ops.ffn_backward(dy, x, wg, wu2, wd, saved, grads=outs[2:], out=outs[1])
    for k, v in zip(("y",) + NAMES, outs):
        check(k, v, want[k])
        assert bool(torch.isnan(v._base[:3]).all()) and bool(torch.isnan(v._base[3:].view(v.shape[0], -1)[:, v.shape[1]:]).all()), k


# rows of equal stride, but only one weight of the pair starts off 16 bytes: both have to come to the same place
@pytest.mark.parametrize("T", [5, 70, 140])
@pytest.mark.parametrize("shifts", [(3, 0), (0, 3), (8, 5)])
def test_ffn_one_unaligned_weight(ops, T, shifts):
    x, wg, wu, wd, dy = ffn_inputs(12, T, 72, 104, torch.bfloat16)
    wide = []
    for i, (w, shift) in enumerate(zip((wg, wu), shifts)):
        wide.append(normal(gen(i), 104, 72, torch.bfloat16, 1.0, 16, shift))
        wide[-1].copy_(w)
    inputs = (x, wide[0], wide[1], wd, dy)
    want = formula(*inputs[:4], "silu", inputs[4])
    for k, v in ffn_both(ops, inputs, "silu").items():
        check(k, v, want[k])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_ffn_large_tiles(ops, dtype):
    inputs = ffn_inputs(5, 3590, 3592, 3608, dtype)
    want = formula(*inputs[:4], "silu", inputs[4])
    for k, v in ffn_both(ops, inputs, "silu").items():
        check(k, v, want[k])


def test_ffn_offsets_beyond_32_bits(ops):
    T, D, F, dtype = 131080, 64, 16392, torch.float16
    x, wg, wu, wd, dy = ffn_inputs(7, T, D, F, dtype)
    got = ffn_both(ops, (x, wg, wu, wd, dy), "silu")
    sums = None
    for at in range(0, T, 16384):
        s = slice(at, min(at + 16384, T))
        part = formula(x[s], wg, wu, wd, "silu", dy[s])
        for k in ("y", "dx"):
            check(k, got[k][s], part[k])
        part = {k: part[k] for k in NAMES[1:]}
        sums = part if sums is None else {k: tuple(a + b for a, b in zip(sums[k], part[k])) for k in part}
    for k in NAMES[1:]:
        value, var = sums[k]
        check(k, got[k], (value, var * 10))                                # float32 sums of T terms were allowed for 16,384 only


# the longest rows that the tiles take: 2^22 elements, of x and the weights, or of dg and du side by side
@pytest.mark.parametrize("shape", [(130, 1 << 22, 64), (130, 64, 1 << 21)])
def test_ffn_longest_rows(ops, shape):
    inputs = ffn_inputs(6, *shape, torch.bfloat16)
    want = formula(*inputs[:4], "silu", inputs[4])
    for k, v in ffn_both(ops, inputs, "silu").items():
        check(k, v, want[k])


# more tokens than tiles of 128 x 128 can be counted for in one launch
def test_ffn_more_tokens_than_small_tiles_reach(ops):
    T, D, F, dtype = (1 << 30) + 77, 8, 8, torch.bfloat16
    _, wg, wu, wd, _ = ffn_inputs(8, 1, D, F, dtype)
    x = torch.empty((T, D), dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=gen(8))
    y = ops.ffn_forward(x, wg, wu, wd)
    for at in (0, (1 << 29) - 500, (1 << 30) - 500, T - 1000):
        s = slice(at, at + 1000)
        check("y", y[s], formula(x[s], wg, wu, wd, "silu")["y"])


def test_ffn_accumulates(ops):
    T, D, F, dtype = 100, 136, 72, torch.bfloat16
    a, b = ffn_inputs(1, T, D, F, dtype), ffn_inputs(2, T, D, F, dtype)
    b = (b[0],) + a[1:4] + (b[4],)
    wa, wb = formula(*a[:4], "silu", a[4]), formula(*b[:4], "silu", b[4])
    for gd in (torch.float32, dtype):
        shapes = ((F, D), (F, D), (D, F))
        grads = [torch.full(s, float("nan"), dtype=gd, device="cuda") for s in shapes]
        ffn_both(ops, a, "silu", grads=grads)                              # written over
        first = [g.clone() for g in grads]
        ffn_both(ops, b, "silu", grads=grads, accumulate=True)
        for k, g, f in zip(NAMES[1:], grads, first):
            check(k, f, wa[k])
            check(k, g, (f.double() + wb[k][0], wb[k][1] + (ACC * f.double()) ** 2))


# What is kept between the passes must not lean to one side.  All values are positive, so that a lean adds up and the roundings do not: of 65,536 x 64
# roundings of h, du or dg to 11 bits a mean of 2^-12 / sqrt(3) / 2^11 is left, six times that 4e-7; the float32 sums (2,048 additions each, 4,096 of
# them) leave less, and the activation's instructions are right to 2^-22.  2^-19 is allowed; values cut to 16 bits lean by 1.1e-5 and more.
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_ffn_float32_gradients_of_many_tokens_lean_to_no_side(ops, act):
    T, D, F, dtype = 65536, 64, 64, torch.float16
    x, wg, wu, wd, dy = (torch.rand(s, generator=gen(30 + i), device="cuda") for i, s in enumerate(((T, D), (F, D), (F, D), (D, F), (T, D))))
    x, wg, wu, wd, dy = [t.to(dtype) for t in (x + 0.25, wg * 4 / D, wu * 4 / D, wd / D, dy + 0.25)]
    grads = [torch.empty(s, device="cuda") for s in ((F, D), (F, D), (D, F))]
    ffn_both(ops, (x, wg, wu, wd, dy), act, grads=grads)
    want = formula(x, wg, wu, wd, act, dy)
    for k, got in zip(NAMES[1:], grads):
        value = want[k][0]
        assert abs(float((got.double() - value).sum() / value.sum())) <= 2.0 ** -19, k


@pytest.mark.parametrize("T", [4, 80])
def test_ffn_bits_repeat_and_streams(ops, T):
    inputs = ffn_inputs(9, T, 264, 520, torch.bfloat16)
    want = ffn_both(ops, inputs, "silu")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y, saved = ops.ffn_forward(*inputs[:4], save=True, stream=side)
    grads = ops.ffn_backward(inputs[4], *inputs[:4], saved, stream=side.cuda_stream)
    side.synchronize()
    for k, v in zip(("y",) + NAMES, (y,) + grads):
        assert torch.equal(v, want[k]), k


def test_ffn_gradients_against_differences(ops):
    T, D, F, dtype, eps = 70, 40, 48, torch.float16, 1e-5
    inputs = ffn_inputs(21, T, D, F, dtype)
    got = ffn_both(ops, inputs, "gelu")
    want = formula(*inputs[:4], "gelu", inputs[4])
    wide = [t.double() for t in inputs]

    def loss(i, d):
        x, wg, wu, wd = [t + d if j == i else t for j, t in enumerate(wide[:4])]
        return float((((act_of("gelu", x @ wg.T)[0] * (x @ wu.T)) @ wd.T) * wide[4]).sum())

    for i, k in enumerate(NAMES):
        v = torch.randn(wide[i].shape, generator=gen(i), device="cuda", dtype=torch.float64)
        slope = (loss(i, eps * v) - loss(i, -eps * v)) / (2 * eps)
        own = float((got[k].double() * v).sum())
        sd = math.sqrt(float(((want[k][1] + (U[dtype] * want[k][0]) ** 2) * v * v).sum()))
        assert abs(slope - own) <= 6 * sd + 1e-5 * abs(slope), (k, slope, own, sd)


@pytest.mark.parametrize("T", [2, 67])
def test_ffn_infinities_and_nans_stay_in_their_rows(ops, T):
    inputs = ffn_inputs(4, T, 72, 77, torch.bfloat16)
    clean = ffn_both(ops, inputs, "silu")
    inputs[0][1, 3] = float("nan")
    inputs[4][1, 5] = float("inf")
    got = ffn_both(ops, inputs, "silu")
    rest = [i for i in range(T) if i != 1]
    assert bool(torch.isnan(got["y"][1]).all()) and bool(torch.isnan(got["dx"][1]).all())
    for k in ("y", "dx"):
        assert torch.equal(got[k][rest], clean[k][rest]), k
    inputs[0][1, 3] = 0.0                                                  # an infinite gradient alone
    inputs[3].abs_()
    inputs[0][1].zero_()                                                   # g = u = 0: dg = dh u act' is not a number, du = dh act(0) too
    got = ffn_both(ops, inputs, "silu")
    assert bool(torch.isnan(got["dx"][1]).all()) and bool(torch.isfinite(got["y"]).all())


def test_ffn_no_tokens(ops):
    inputs = ffn_inputs(4, 0, 16, 24, torch.bfloat16)
    got = ffn_both(ops, inputs, "silu")
    assert got["y"].shape == (0, 16) and got["dx"].shape == (0, 16)
    for k in NAMES[1:]:
        assert bool((got[k] == 0).all())


# odd widths, strides that differ: what a packing would read and copy
def test_ffn_no_tokens_at_odd_widths(ops):
    from paper_2508_21613_amd import binding as B
    D, F = 65, 97
    x, wg, wu, wd, dy = ffn_inputs(4, 0, D, F, torch.bfloat16)
    wu = normal(gen(1), F, D, torch.bfloat16, 1.0, 2)
    y, saved = ops.ffn_forward(x, wg, wu, wd, save=True)
    assert y.shape == (0, D)
    grads = [torch.full(s, 7.0, device="cuda") for s in ((F, D), (F, D), (D, F))]
    ops.ffn_backward(dy, x, wg, wu, wd, saved, grads=grads, accumulate=True)
    assert all(bool((t == 7).all()) for t in grads)
    assert ops.ffn_backward(dy, x, wg, wu, wd, saved, grads=grads)[0].shape == (0, D)
    assert all(bool((t == 0).all()) for t in grads)
    # inputs, results for tokens and scratch may be missing altogether
    grads = [torch.full(s, 7.0, device="cuda") for s in ((F, D), (F, D), (D, F))]
    d = B.Ffn(1, 0, 0, D, F, None, None, None, None, D, D, D + 2, F)
    g = B.FfnGradients(None, None, *(t.data_ptr() for t in grads), D, D, D, D, F, 0, 0)
    assert B.lib().chm_ffn_backward(d, g, None, 0, torch.cuda.current_stream().cuda_stream) == B.OK
    assert all(bool((t == 0).all()) for t in grads)


# ------------------------------------------------------------------------------------------------ embedding
def lookup_want(tokens, table, scale):
    live = (tokens >= 0) & (tokens < table.shape[0])
    rows = torch.zeros((len(tokens), table.shape[1]), dtype=torch.float64, device="cuda")
    rows[live] = table[tokens[live].long()].double() * scale
    return rows


def gradient_want(dy, tokens, V, scale):
    live = (tokens >= 0) & (tokens < V)
    order = tokens[live].long()
    v = torch.zeros((V, dy.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, order, dy[live].double() * scale)
    counts = torch.bincount(order, minlength=V)[:, None].double()
    sq = torch.zeros_like(v).index_add_(0, order, (dy[live].double() * scale) ** 2)
    return v, ACC ** 2 * (counts + 2) * sq


EMBED = [(1, 1, 1), (1, 5, 64), (7, 3, 9), (255, 40, 31), (256, 100, 515), (257, 100, 515), (300, 7, 64), (511, 60, 9), (512, 300, 70), (513, 300, 70), (1000, 1, 72), (1024, 33, 8), (2049, 5000, 100),
         (4096, 100, 2049), (5000, 513, 130), (16384, 3000, 72), (16385, 511, 40), (40000, 70000, 24), (70001, 129, 16)]


def make_tokens(seed, n, V, index, kind):
    g = gen(seed)
    if kind == "same":
        t = torch.full((n,), V - 1, device="cuda")
    elif kind == "none":
        t = torch.full((n,), -1, device="cuda")
    else:
        t = (torch.rand(n, generator=g, device="cuda").double() ** 3 * V).long().clamp_(0, V - 1)
        if kind == "outside":                                              # of another shard, padding, far outside
            k = torch.rand(n, generator=g, device="cuda")
            t = torch.where(k < 0.15, -1 - t, torch.where(k < 0.3, t + V, t))
            t[:: 97] = -(1 << 31) if index == torch.int32 else -(1 << 62)
            t[5:: 97] = (1 << 31) - 1 if index == torch.int32 else (1 << 32) + V - 1
    return t.to(index)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("kind", ["some", "outside"])
@pytest.mark.parametrize("shape", EMBED)
def test_embedding(ops, shape, kind, dtype):
    n, V, D = shape
    index = (torch.int32, torch.int64)[(n + V) % 2]
    pad, shift = ((0, 0), (3, 1), (8, 8))[(n + D) % 3]
    g = gen(n + V)
    tokens, scale = make_tokens(n, n, V, index, kind), 1.75
    table, dy = normal(g, V, D, dtype, 1.0, pad, shift), normal(g, n, D, dtype, 1.0, pad, shift)
    rows = lookup_want(tokens, table, scale)
    check("rows", ops.embedding_lookup(tokens, table, scale), (rows, torch.zeros_like(rows)))
    want = gradient_want(dy, tokens, V, scale)
    got = ops.embedding_gradient(dy, tokens, V, scale)
    check("dtable", got, want)
    assert bool((got[want[1].amax(1) == 0] == 0).all())                    # rows that no token names
    assert torch.equal(got, ops.embedding_gradient(dy, tokens, V, scale))
    for gd in {dtype, torch.float32}:
        start = normal(g, V, D, gd, 1.0, pad, shift)
        out = normal(g, V, D, gd, 1.0, pad, shift)
        out.copy_(start)
        ops.embedding_gradient(dy, tokens, scale=scale, out=out, accumulate=True)
        check("added", out, (want[0] + start.double(), want[1] + (ACC * start.double()) ** 2))
        named = torch.zeros(V, dtype=torch.bool, device="cuda")
        named[tokens[(tokens >= 0) & (tokens < V)].long()] = True
        assert torch.equal(out[~named], start[~named])
        if pad:
            assert bool(torch.isnan(out._base[:shift]).all()) and bool(torch.isnan(out._base[shift:].view(V, -1)[:, D:]).all())


@pytest.mark.parametrize("kind", ["same", "none"])
@pytest.mark.parametrize("n", [1, 200, 500, 3000, 20000])
def test_embedding_one_token_or_none(ops, n, kind):
    V, D = 37, 100
    tokens, dy = make_tokens(1, n, V, torch.int64, kind), normal(gen(2), n, D, torch.float32)
    check("dtable", ops.embedding_gradient(dy, tokens, V), gradient_want(dy, tokens, V, 1.0))


def test_embedding_empty(ops):
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    table = normal(gen(1), 10, 6, torch.bfloat16)
    assert ops.embedding_lookup(none, table).shape == (0, 6)
    out = ops.embedding_gradient(torch.empty((0, 6), dtype=torch.bfloat16, device="cuda"), none, 10)
    assert out.shape == (10, 6) and bool((out == 0).all())
    assert bool((ops.embedding_lookup(torch.zeros(3, dtype=torch.int64, device="cuda"), table[:0]) == 0).all())


def test_embedding_offsets_beyond_32_bits(ops):
    V, D = 600000, 4096
    tokens = torch.tensor([V - 1, 0, V - 1, 530000, -1], device="cuda")
    table = torch.zeros((V, D), dtype=torch.bfloat16, device="cuda")
    table[V - 1], table[530000], table[0] = 3, 5, 7
    got = ops.embedding_lookup(tokens, table)
    assert [float(v) for v in got[:, D - 1]] == [3, 7, 3, 5, 0] and bool((got == got[:, :1]).all())
    for n in (5, 300):
        t = tokens.repeat(n // 5)
        dy = torch.ones((n, D), dtype=torch.bfloat16, device="cuda")
        table.fill_(9)
        ops.embedding_gradient(dy, t, out=table)
        k = n // 5
        for row, value in ((V - 1, 2 * k), (0, k), (530000, k), (1, 0), (V - 2, 0), (300000, 0), (530001, 0)):
            assert bool((table[row] == value).all()), (n, row)


# rows and places that one launch of a workgroup each cannot count: 2^32 threads
@pytest.mark.parametrize("n", [300, 1000])
def test_embedding_gradient_of_more_rows_than_a_grid_holds(ops, n):
    V = (1 << 29) + 45
    tokens = torch.tensor([V - 1, 0, 1 << 25, (1 << 25) - 1, V - 1, 400000001, -1, V], device="cuda").repeat((n + 7) // 8)[:n]
    dy = torch.ones((n, 1), dtype=torch.bfloat16, device="cuda")
    out = torch.full((V, 1), 9.0, dtype=torch.bfloat16, device="cuda")
    ops.embedding_gradient(dy, tokens, out=out)
    for row in (V - 1, 0, 1 << 25, (1 << 25) - 1, 400000001):
        assert float(out[row]) == float((tokens == row).sum()), row
        out[row] = 0
    assert bool((out == 0).all())


def test_embedding_lookup_of_more_places_than_a_grid_holds(ops):
    n, V = (1 << 30) + 4099, 251
    tokens = torch.arange(n, dtype=torch.int32, device="cuda") % (V + 1)                # the last one is outside the table
    table = torch.arange(1, V + 1, device="cuda").bfloat16()[:, None]
    got = ops.embedding_lookup(tokens, table)
    want = torch.cat([table[:, 0], torch.zeros(1, dtype=table.dtype, device="cuda")])
    for at in range(0, n, 1 << 28):
        s = slice(at, min(at + (1 << 28), n))
        assert torch.equal(got[s, 0], want[tokens[s].long()]), at


def test_embedding_infinities_stay_in_their_rows(ops):
    for n in (100, 1000):
        tokens = torch.arange(n, device="cuda") % 50
        dy = torch.ones((n, 40), dtype=torch.bfloat16, device="cuda")
        dy[3, 7], dy[4, 8] = float("inf"), float("nan")
        got = ops.embedding_gradient(dy, tokens, 60)
        assert float(got[3, 7]) == float("inf") and bool(torch.isnan(got[4, 8]))
        got[3, 7] = got[4, 8] = n // 50
        assert bool((got[:50] == n // 50).all()) and bool((got[50:] == 0).all())


# ------------------------------------------------------------------------------------------------ norm and clipping
def clip_want(grads, max_norm, sumsq=None):
    total = sum(float((g.double() ** 2).sum()) for g in grads) if sumsq is None else sumsq
    norm = math.sqrt(total)
    return norm, min(1.0, max_norm / (norm + 1e-6))


def check_clip(norm, got, grads, max_norm, sumsq=None):
    n, c = clip_want(grads, max_norm, sumsq)
    assert norm.dtype == torch.float32 and norm.dim() == 0
    assert abs(float(norm) - n) <= 2 * 2.0 ** -24 * n
    for a, g in zip(got, grads):
        w = g.double() * c
        # the factor is off by a few float32 roundings, then one rounding to the gradient's type
        check("clipped", a, (w, (4 * ACC * w) ** 2))


CLIP = [[1], [5, 0, 3], [8191, 8192, 8193], [1 << 20, 1, 77777], [3] * 300, [100003] * 40, [(1 << 22) + 5]]


@pytest.mark.parametrize("factor", [0.3, 4.0])
@pytest.mark.parametrize("sizes", CLIP, ids=lambda s: "%dx%d" % (len(s), s[0]))
def test_clip(ops, sizes, factor):
    g = gen(len(sizes))
    types = (torch.float32, torch.bfloat16, torch.float16)
    grads = []
    for i, n in enumerate(sizes):
        shift = i % 5
        buf = torch.empty(n + shift + 3, dtype=types[(i + len(sizes)) % 3], device="cuda")
        buf.copy_(torch.randn(buf.shape, generator=g, device="cuda"))
        grads.append(buf[shift:shift + n])
    raw = [t.clone() for t in grads]
    rims = [t._base.clone() for t in grads]
    max_norm = factor * clip_want(raw, 1.0)[0]
    out = [torch.full_like(t, 99.0) for t in grads]
    with_out = ops.Gradients(grads, out)
    norm = with_out.clip(max_norm)
    check_clip(norm, out, raw, max_norm)
    assert all(torch.equal(a, b) for a, b in zip(grads, raw))
    here = ops.Gradients(grads)
    total = here.sumsq()
    assert total.dtype == torch.float64 and abs(float(total) - clip_want(raw, 1.0)[0] ** 2) <= 1e-12 * float(total) + 1e-300
    assert torch.equal(here.clip(max_norm), norm)
    assert all(torch.equal(a, b) for a, b in zip(grads, out))
    for t, rim in zip(grads, rims):                                        # nothing beside the tensors is written
        mine = t._base.clone()
        at = t.storage_offset()
        mine[at:at + t.numel()] = rim[at:at + t.numel()]
        assert torch.equal(mine, rim)
    here.close()
    with_out.close()


def test_clip_with_the_sum_of_other_stages(ops):
    a, b = [normal(gen(1), 30, 70, torch.float32)], [normal(gen(2), 9, 1000, torch.bfloat16), normal(gen(3), 3, 3, torch.float32)]
    raw = [t.clone() for t in a + b]
    sa, sb = ops.Gradients(a), ops.Gradients(b)
    total = sa.sumsq() + sb.sumsq()
    norms = [sa.clip(0.5, sumsq=total), sb.clip(0.5, sumsq=total)]
    for norm in norms:
        check_clip(norm, a + b, raw, 0.5)


def test_clip_refuses_results_over_other_tensors(ops):
    from paper_2508_21613_amd import binding as B
    buf = normal(gen(1), 1, 1000, torch.float32)[0]
    other = torch.zeros(1000, device="cuda")
    a, b = buf[:600], buf[600:]
    for grads, out in (([a, b], None), ([a, b], [other[:600], other[600:]]), ([a, a], [other[:600], torch.zeros(600, device="cuda")]), ([b[:0], a, a[:0]], None)):
        raw = [t.clone() for t in grads]
        check_clip(ops.Gradients(grads, out).clip(0.5), out or grads, raw, 0.5)
    for grads, out in (([a, a], None), ([a, buf[599:]], None), ([buf, a[5:9]], None), ([a, b], [other[:600], other[599:999]]), ([a, b], [b[:0].new_zeros(600), a[:400]]),
                       ([a], [buf[1:601]])):
        raw = buf.clone()
        g = ops.Gradients(grads, out)
        want = sum(float((t.double() ** 2).sum()) for t in grads)
        assert abs(float(g.sumsq()) - want) <= 1e-12 * want                # reading is no harm
        with pytest.raises(B.ChmError) as e:
            g.clip(0.5)
        assert e.value.code == B.ERR_ARG and torch.equal(buf, raw)


def test_saved_has_to_be_one_stretch_of_memory(ops):
    from paper_2508_21613_amd import binding as B
    x, wg, wu, wd, dy = ffn_inputs(15, 20, 64, 64, torch.bfloat16)
    y, saved = ops.ffn_forward(x, wg, wu, wd, save=True)
    for other in (saved.repeat_interleave(2)[::2], saved[:1].expand(saved.shape)):     # as many elements, elsewhere in memory or nowhere
        with pytest.raises(B.ChmError) as e:
            ops.ffn_backward(dy, x, wg, wu, wd, other)
        assert e.value.code == B.ERR_ARG
    assert torch.equal(ops.ffn_backward(dy, x, wg, wu, wd, saved.clone())[0], ops.ffn_backward(dy, x, wg, wu, wd, saved)[0])


def test_gradients_are_not_lost_without_a_word(ops):
    from paper_2508_21613_amd import binding as B
    inputs = ffn_inputs(16, 20, 64, 64, torch.bfloat16)
    x, wg, wu, wd, dy = inputs
    tokens = torch.arange(20, device="cuda")
    want, row = ops.ffn_forward(x, wg, wu, wd), ops.embedding_lookup(tokens, wg)
    for t in inputs[:4]:
        t.requires_grad_()
        calls = [lambda: ops.ffn_forward(x, wg, wu, wd)] + ([lambda: ops.embedding_lookup(tokens, wg)] if t is wg else [])
        for call in calls:
            with pytest.raises(B.ChmError) as e:
                call()
            assert e.value.code == B.ERR_ARG and "no_grad" in str(e.value)
        with torch.no_grad():
            assert torch.equal(ops.ffn_forward(x, wg, wu, wd), want) and torch.equal(ops.embedding_lookup(tokens, wg), row)
        y, saved = ops.ffn_forward(x, wg, wu, wd, save=True)               # a caller that takes the gradients by the calls for them
        assert torch.equal(y, want) and not y.requires_grad and not ops.ffn_backward(dy, x, wg, wu, wd, saved)[0].requires_grad
        t.requires_grad_(False)


def test_results_over_inputs(ops):
    from paper_2508_21613_amd import binding as B
    for T in (5, 100):
        x, wg, wu, wd, dy = ffn_inputs(14, T, 64, 64, torch.bfloat16)
        want = ops.ffn_forward(x, wg, wu, wd)
        y, saved = ops.ffn_forward(x, wg, wu, wd, save=True)
        for call in (lambda: ops.ffn_backward(dy, x, wg, wu, wd, saved, out=dy), lambda: ops.ffn_backward(dy, x, wg, wu, wd, saved, out=x),
                     lambda: ops.ffn_backward(dy, x, wg, wu, wd, saved, grads=(wg, wu, wd)), lambda: ops.ffn_forward(x[:, :], wg, wu, wd, out=wd[:T])):
            with pytest.raises(B.ChmError) as e:
                call()
            assert e.value.code == B.ERR_ARG
        both = normal(gen(1), T, 128, torch.bfloat16)                      # columns of the same rows
        both[:, 64:] = x
        assert torch.equal(ops.ffn_forward(both[:, 64:], wg, wu, wd, out=both[:, :64]), want) and torch.equal(both[:, 64:], x)
        assert torch.equal(ops.ffn_forward(x, wg, wu, wd, out=x), want)    # over x itself
    tokens = torch.arange(8, device="cuda")
    for call in (lambda: ops.embedding_lookup(tokens, wg, out=wg[:8]), lambda: ops.embedding_gradient(dy, torch.arange(100, device="cuda"), out=dy)):
        with pytest.raises(B.ChmError) as e:
            call()
        assert e.value.code == B.ERR_ARG


def test_clip_on_one_stream_after_another(ops):
    """calls share a workspace: one on another stream begins when the one before has ended"""
    t = normal(gen(1), 1000, 1000, torch.float32)
    filler = torch.empty(1 << 28, device="cuda")
    g = ops.Gradients([t], [torch.empty_like(t)])
    want = float(g.clip(1.0))
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for first, second, call in ((a, b, g.sumsq), (b, a, lambda stream: g.clip(1.0, stream=stream)), (a, b, lambda stream: g.clip(1.0, stream=stream.cuda_stream))):
        with torch.cuda.stream(first):
            for _ in range(30):
                filler.zero_()                                             # some 5 ms in all
        one = call(stream=first) if call == g.sumsq else call(first)
        ended = torch.cuda.Event()
        ended.record(first)
        two = g.clip(1.0, stream=second)
        second.synchronize()
        assert ended.query()
        assert float(two) == want and (float(one) == want or call == g.sumsq)
        torch.cuda.synchronize()


def test_gradients_keep_their_memory(ops):
    """a tensor that is given other memory leaves the listed one with the list"""
    t, o = torch.ones(1 << 20, device="cuda"), torch.zeros(1 << 20, device="cuda")
    g, places = ops.Gradients([t], [o]), {t.data_ptr(), o.data_ptr()}
    t.data, o.data = torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda")
    others = [torch.zeros(1 << 20, device="cuda") for _ in range(4)]
    assert not places & {k.data_ptr() for k in others}
    assert float(g.clip(1.0)) == 1024.0 and all(bool((k == 0).all()) for k in others)


def test_clip_in_any_dense_layout(ops):
    t = torch.randn(40, 50, generator=gen(1), device="cuda").t()
    raw = t.clone()
    norm = ops.Gradients([t]).clip(0.1)
    check_clip(norm, [t], [raw], 0.1)


def test_clip_range_of_values(ops):
    big = torch.full((1000,), 1e30, device="cuda")                         # squares beyond float32, and below it
    small = torch.full((1000,), 1e-30, device="cuda")
    for t in (big, small):
        raw = t.clone()
        norm = ops.Gradients([t]).clip(float(raw[0]))
        check_clip(norm, [t], [raw], float(raw[0]))
    for bad in (float("inf"), float("nan")):
        t = torch.ones(3000, device="cuda")
        t[2999] = bad
        norm = ops.Gradients([t]).clip(1.0)
        assert not bool(torch.isfinite(norm)) and bool(torch.isnan(t[2999]))
        if bad == float("inf"):
            assert float(norm) == bad and bool((t[:2999] == 0).all())      # 1 / infinity
        else:
            assert bool(torch.isnan(t).all())
    t = torch.ones(4, device="cuda")
    assert float(ops.Gradients([t]).clip(0.0)) == 2.0 and bool((t == 0).all())
    zero = torch.zeros(4, device="cuda")
    assert float(ops.Gradients([zero]).clip(1.0)) == 0.0 and bool((zero == 0).all())
    assert float(ops.Gradients([]).clip(1.0)) == 0.0 and float(ops.Gradients([zero[:0]]).sumsq()) == 0.0


def test_clip_by_a_norm_beyond_float32(ops):
    """the gradients are finite: so is the factor, whatever the returned norm's type holds"""
    t = torch.full((1000,), 3e38, device="cuda")
    raw = t.clone()
    norm = ops.Gradients([t]).clip(1000.0)
    want = clip_want([raw], 1000.0)[1] * raw.double()
    assert float(norm) == math.inf
    check("clipped", t, (want, (4 * ACC * want) ** 2))


def test_clip_lengths_beyond_32_bits(ops):
    n = (1 << 31) + 5
    t = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    t[n - 1] = 2.0
    norm = ops.Gradients([t]).clip(0.5 * math.sqrt(n + 3.0))
    assert abs(float(norm) - math.sqrt(n + 3.0)) <= 2.0 ** -23 * float(norm)
    assert bool((t[:n - 1] == 0.5).all()) and float(t[n - 1]) == 1.0


# ------------------------------------------------------------------------------------------------ all of them
def test_a_captured_step_replays(ops):
    T, D, F, V, dtype = 300, 128, 264, 500, torch.bfloat16
    _, wg, wu, wd, dy = ffn_inputs(31, T, D, F, dtype)
    table = normal(gen(3), V, D, dtype)
    tokens = make_tokens(4, T, V, torch.int64, "outside")
    grads = [torch.zeros(s, device="cuda") for s in ((F, D), (F, D), (D, F), (V, D))]
    clipped = [torch.zeros_like(t) for t in grads]
    lists = ops.Gradients(grads, clipped)

    def step():
        x = ops.embedding_lookup(tokens, table, 2.0)
        y, saved = ops.ffn_forward(x, wg, wu, wd, save=True)
        dx = ops.ffn_backward(dy, x, wg, wu, wd, saved, grads=grads[:3])[0]
        ops.embedding_gradient(dx, tokens, scale=2.0, out=grads[3])
        return y, lists.clip(0.1)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, norm = step()
    for seed in range(4):
        dy.copy_(torch.randn(T, D, generator=gen(seed), device="cuda"))
        tokens.copy_(make_tokens(seed, T, V, torch.int64, "outside"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in [y, norm] + grads + clipped]
        want_y, want_norm = step()
        torch.cuda.synchronize()
        for a, b in zip(got, [want_y, want_norm] + grads + clipped):
            assert torch.equal(a, b)


def test_refusals(ops):
    from paper_2508_21613_amd import binding as B
    x, wg, wu, wd, dy = ffn_inputs(1, 4, 16, 24, torch.bfloat16)
    saved = ops.ffn_forward(x, wg, wu, wd, save=True)[1]
    tokens = torch.zeros(4, dtype=torch.int64, device="cuda")
    grad = torch.zeros(8, device="cuda")
    calls = [lambda: ops.ffn_forward(x.float(), wg, wu, wd), lambda: ops.ffn_forward(x, wg.half(), wu, wd), lambda: ops.ffn_forward(x.cpu(), wg, wu, wd),
             lambda: ops.ffn_forward(x, wg[:, :8], wu, wd), lambda: ops.ffn_forward(x, wg, wu[:20], wd), lambda: ops.ffn_forward(x, wg, wu, wd.t()),
             lambda: ops.ffn_forward(x[0], wg, wu, wd), lambda: ops.ffn_forward(x, wg, wu, wd, activation="relu"),
             lambda: ops.ffn_forward(x[:1].expand(4, 16), wg, wu, wd), lambda: ops.ffn_forward(x, wg, wu, wd, out=dy.float()),
             lambda: ops.ffn_forward(x, wg.t().contiguous().t(), wu, wd), lambda: ops.ffn_forward(x[:, :0], wg[:, :0], wu[:, :0], wd[:0]),
             lambda: ops.ffn_backward(dy[:3], x, wg, wu, wd, saved), lambda: ops.ffn_backward(dy, x, wg, wu, wd, saved[:100]),
             lambda: ops.ffn_backward(dy, x, wg, wu, wd, saved, accumulate=True), lambda: ops.ffn_backward(dy, x, wg, wu, wd, None),
             lambda: ops.ffn_backward(dy, x, wg, wu, wd, saved, grads=[wg.half(), wu.half(), wd.half()]),
             lambda: ops.ffn_backward(dy, x, wg, wu, wd, saved, grads=[wg.clone(), wu.clone()]),
             lambda: ops.ffn_backward(dy, x, wg, wu, wd, saved, grads=[torch.zeros((24, 20), dtype=x.dtype, device="cuda")[:, :16], wu.clone(), wd.clone()]),
             lambda: ops.embedding_lookup(tokens.short(), wg), lambda: ops.embedding_lookup(tokens.cpu(), wg), lambda: ops.embedding_lookup(tokens, wg.double()),
             lambda: ops.embedding_lookup(tokens, wg, out=torch.zeros((3, 16), dtype=wg.dtype, device="cuda")),
             lambda: ops.embedding_gradient(dy, tokens[:3], 9), lambda: ops.embedding_gradient(dy, tokens), lambda: ops.embedding_gradient(dy, tokens, -1),
             lambda: ops.embedding_gradient(dy, tokens, 9, accumulate=True), lambda: ops.embedding_gradient(dy, tokens, out=wg.half()),
             lambda: ops.embedding_gradient(dy, tokens, 9, out=wg),
             lambda: ops.Gradients([grad.cpu()]), lambda: ops.Gradients([grad.double()]), lambda: ops.Gradients([grad[::2]]),
             lambda: ops.Gradients([grad], [grad.half()]), lambda: ops.Gradients([grad], []), lambda: ops.Gradients([grad]).clip(-1.0),
             lambda: ops.Gradients([grad]).clip(float("nan")), lambda: ops.Gradients([grad]).clip(1.0, sumsq=grad)]
    for i, call in enumerate(calls):
        with pytest.raises(B.ChmError) as e:
            call()
        assert e.value.code == B.ERR_ARG, i
    d = ops._ffn(x, wg, wu, wd, "silu")[0]                                 # scratch that is too short
    ws = torch.empty(64, dtype=torch.uint8, device="cuda")
    assert B.lib().chm_ffn_forward(d, dy.data_ptr(), 16, ws.data_ptr(), 64, None) == B.ERR_LIMIT
