"""What the operators' entry points answer without a GPU: sizes of workspaces and refusals."""
import ctypes as C

import pytest
import torch

from paper_2508_21613_amd import binding as B
from paper_2508_21613_amd import operators as ops


def _ffn(T=100, D=64, F=96, **kw):
    d = B.Ffn(dtype=1, activation=0, tokens=T, width=D, features=F, ld_x=D, ld_gate=D, ld_up=D, ld_down=F)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _grads(T=100, D=64, F=96, **kw):
    g = B.FfnGradients(ld_dy=D, ld_dx=D, ld_dw_gate=D, ld_dw_up=D, ld_dw_down=F, grad_dtype=1)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def _sizes(d, g=None):
    out = [C.c_uint64() for _ in range(3)]
    rc = B.lib().chm_ffn_sizes(d, g, *out)
    return rc, [int(v.value) for v in out]


def test_ffn_sizes():
    rc, (saved, forward, backward) = _sizes(_ffn(), _grads())
    assert rc == B.OK and saved == 112 * 96 * 6 and forward >= 100 * 96 * 2 and backward >= 100 * 96 * 6
    assert _sizes(_ffn())[1][2] == 0
    assert _sizes(_ffn(F=97, ld_down=97))[1][0] == 112 * 128 * 6                       # blocks of 16 x 32
    even, odd = _sizes(_ffn(), _grads())[1], _sizes(_ffn(ld_gate=65, ld_up=65), _grads())[1]
    assert odd[1] >= even[1] + 2 * 96 * 64 * 2 and odd[2] >= even[2] + 2 * 96 * 64 * 2  # packed copies of both weights
    assert _sizes(_ffn(T=0), _grads(T=0))[0] == B.OK


def test_ffn_packs_both_weights_of_a_product_or_none():
    """the tiles take both at one row length: a weight that starts off 16 bytes takes the other one with it"""
    plain = _sizes(_ffn(ld_gate=72, ld_up=72), _grads())[1]
    copy = 96 * 64 * 2
    for one in (dict(w_gate=8), dict(w_up=8), dict(w_gate=8, w_up=2), dict(ld_up=80)):
        both = _sizes(_ffn(**dict(dict(ld_gate=72, ld_up=72), **one)), _grads())[1]
        assert both[1] == plain[1] + 2 * copy and both[2] == plain[2] + 2 * copy, one


def test_ffn_without_tokens_packs_nothing():
    """no operand need be there then: a packing would read the weights, wherever their pointers lead"""
    d = _ffn(T=0, D=65, F=97, ld_x=65, ld_gate=65, ld_up=67, ld_down=97)
    g = _grads(T=0, ld_dy=65, ld_dx=65, ld_dw_gate=65, ld_dw_up=65, ld_dw_down=97)
    assert _sizes(d, g) == (B.OK, [0, 0, 0])
    g.dw_gate = g.dw_up = g.dw_down = 64                                                # never touched: nothing is added
    g.accumulate = 1
    assert B.lib().chm_ffn_backward(d, g, None, 0, None) == B.OK


def test_ffn_rows_that_the_tiles_cannot_reach_are_refused():
    """offsets within a tile are of 32 bits: up to 2^22 elements a row, of which dg and du take two of `features`"""
    def sizes(T, D, F):
        d, g = _ffn(T, D, F), _grads(T, D, F)
        some = [C.c_uint64() for _ in range(2)]
        return B.lib().chm_ffn_sizes(d, None, *some, None), B.lib().chm_ffn_sizes(d, g, some[0], None, some[1])

    W, H = 1 << 22, 1 << 21
    assert sizes(128, W, 64) == sizes(128, 64, H) == sizes(8, W, H) == (B.OK, B.OK)
    assert sizes(128, W + 8, 64) == sizes(128, 64, H + 8) == sizes(256, 64, 8454664) == (B.ERR_ARG, B.ERR_ARG)
    assert sizes(8, 1 << 24, 1 << 24) == sizes(1, W + 8, 8) == (B.OK, B.ERR_ARG)        # few tokens count in 64 bits
    assert sizes(0, 1 << 24, 1 << 24) == (B.OK, B.OK)
    for D, F in ((W + 8, 64), (64, H + 8)):
        assert B.lib().chm_ffn_forward(_ffn(128, D, F), None, D, None, 0, None) == B.ERR_ARG
        one = _grads(128, D, F, dw_gate=64, dw_up=64, dw_down=64)
        assert B.lib().chm_ffn_backward(_ffn(128, D, F), one, None, 0, None) == B.ERR_ARG


def test_ffn_launches_fit_a_grid():
    """a launch has fewer than 2^32 threads: the largest tiles reach up to 2^31 - 2^13 tokens, and what none reaches is refused"""
    L, any_ = B.lib(), dict(x=64, w_gate=64, w_up=64, w_down=64)
    for T, F, rc in (((1 << 31) - 1, 8, B.ERR_ARG), ((1 << 31) - 8193, 8, B.ERR_LIMIT), (1 << 30, 8, B.ERR_LIMIT), (1 << 30, 4096, B.ERR_ARG)):
        assert L.chm_ffn_forward(_ffn(T, 8, F, **any_), 64, 8, 64, 1, None) == rc, T     # ERR_LIMIT: taken, but the scratch is too short
        g = _grads(T, 8, F, dy=64, dx=64, dw_gate=64, dw_up=64, dw_down=64)
        assert L.chm_ffn_backward(_ffn(T, 8, F, saved=64, **any_), g, 64, 1, None) == rc, T


@pytest.mark.skipif(torch.cuda.is_available(), reason="pointers that nobody may follow")
def test_results_over_other_tensors_are_refused():
    """without a GPU a call that goes on to its launches says ERR_HIP"""
    L, T, D, F, M = B.lib(), 100, 64, 96, 1 << 20
    at = {k: (i + 1) * M for i, k in enumerate(("x", "w_gate", "w_up", "w_down", "saved", "dy", "dx", "dw_gate", "dw_up", "dw_down"))}
    ffn, grad = ("x", "w_gate", "w_up", "w_down", "saved"), ("dy", "dx", "dw_gate", "dw_up", "dw_down")

    def forward(y=20 * M, ld_y=D, scratch=30 * M, **kw):
        return L.chm_ffn_forward(_ffn(T, D, F, **{k: dict(at, **kw)[k] for k in ffn}), y, ld_y, scratch, M, None)

    def backward(scratch=30 * M, ld=None, **kw):
        g = _grads(T, D, F, **{k: dict(at, **kw)[k] for k in grad})
        if ld:
            g.ld_dw_gate = g.ld_dw_up = ld
        return L.chm_ffn_backward(_ffn(T, D, F, **{k: dict(at, **kw)[k] for k in ffn}), g, scratch, M, None)

    assert forward() == forward(y=at["x"]) == forward(y=at["x"] + 2) == B.ERR_HIP         # y may lie over x
    for k in ("w_gate", "w_up", "w_down", "saved"):
        assert forward(y=at[k]) == forward(scratch=at[k]) == B.ERR_ARG, k
    assert forward(saved=at["x"]) == forward(scratch=at["x"]) == forward(y=30 * M) == forward(y=30 * M - 2 * T * D + 2) == B.ERR_ARG
    assert forward(y=30 * M - 2 * T * D) == B.ERR_HIP
    assert backward() == B.ERR_HIP
    for k in grad[1:]:
        for other in ffn + grad:
            if other != k:
                assert backward(**{k: at[other]}) == B.ERR_ARG, (k, other)
    assert backward(dx=at["dy"] + 2 * (T * D - 1)) == B.ERR_ARG and backward(dx=at["dy"] + 2 * T * D) == B.ERR_HIP
    # columns of one buffer
    assert backward(dw_up=at["dw_gate"] + 2 * D, ld=2 * D) == B.ERR_HIP and backward(dw_up=at["dw_gate"] + 2 * D - 2, ld=2 * D) == B.ERR_ARG
    assert backward(dw_up=at["dw_gate"] + 2 * D, ld=2 * D - 1) == B.ERR_ARG

    n, V = 600, 50

    def embedding_gradient(grad=M, dy=2 * M, tokens=3 * M, scratch=4 * M):
        return L.chm_embedding_gradient(1, 1, 64, tokens, n, dy, D, V, D, 1.0, grad, D, 0, scratch, M, None)

    assert embedding_gradient() == embedding_gradient(grad=2 * M - 2 * V * D) == B.ERR_HIP
    for bad in (dict(grad=2 * M), dict(grad=2 * M - 2), dict(grad=3 * M), dict(scratch=2 * M), dict(scratch=3 * M), dict(scratch=M)):
        assert embedding_gradient(**bad) == B.ERR_ARG, bad
    for out in (M, M + 2 * V * D - 2, 3 * M, 3 * M + 8 * n - 2):
        assert L.chm_embedding_lookup(1, 64, 3 * M, n, M, D, V, D, 1.0, out, D, None) == B.ERR_ARG
    assert L.chm_embedding_lookup(1, 64, 3 * M, n, M, D, V, D, 1.0, M + 2 * V * D, D, None) == B.ERR_HIP


def test_rows_that_share_memory(tmp_path):
    """csrc/chm_overlap.h against marking every byte"""
    import os
    import subprocess
    csrc = os.path.join(os.path.dirname(os.path.abspath(B.__file__)), "csrc")
    src = tmp_path / "overlap.cpp"
    src.write_text(r'''
#include "chm_overlap.h"
#include <stdio.h>
#include <string.h>
#include <random>
using chm_overlap::Rows;
int main() {
  std::mt19937 rng(1);
  static char memory[400], mark[400];
  long shared = 0;
  const auto pick = [&](int n) { return (int64_t)(rng() % n); };
  const auto rows = [&]() { Rows r{memory + pick(90), pick(7), pick(9), 0}; r.pitch = r.bytes + (pick(3) ? pick(12) : 0); if (!r.pitch) r.pitch = 1; return r; };
  for (int t = 0; t < 1000000; ++t) {
    const Rows a = rows();
    Rows b = rows();
    if (pick(2) && a.pitch >= b.bytes) b.pitch = a.pitch;
    bool want = false;
    memset(mark, 0, sizeof mark);
    for (int64_t i = 0; i < a.rows; ++i) memset(mark + ((const char *)a.p - memory) + i * a.pitch, 1, a.bytes);
    for (int64_t i = 0; i < b.rows; ++i)
      for (int64_t k = 0; k < b.bytes; ++k) want |= mark[((const char *)b.p - memory) + i * b.pitch + k] != 0;
    if (chm_overlap::share(a, b) != want || chm_overlap::share(b, a) != want) { printf("case %d\n", t); return 1; }
    shared += want;
  }
  return shared > 100000 ? 0 : 2;
}
''')
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", csrc, "-o", str(tmp_path / "overlap"), str(src)], check=True)
    subprocess.run([str(tmp_path / "overlap")], check=True)


@pytest.mark.parametrize("change", [dict(dtype=0), dict(dtype=3), dict(activation=3), dict(activation=-1), dict(tokens=-1), dict(width=0),
                                    dict(features=0), dict(width=1 << 25), dict(ld_x=63), dict(ld_gate=63), dict(ld_up=63), dict(ld_down=95),
                                    dict(x=1), dict(w_down=3), dict(saved=8), dict(ld_x=1 << 32)])
def test_ffn_refusals(change):
    assert _sizes(_ffn(**change))[0] == B.ERR_ARG
    assert B.lib().chm_ffn_forward(_ffn(**change), None, 64, None, 0, None) == B.ERR_ARG
    assert B.lib().chm_ffn_backward(_ffn(**change), _grads(), None, 0, None) == B.ERR_ARG


@pytest.mark.parametrize("change", [dict(grad_dtype=2), dict(grad_dtype=-1), dict(ld_dy=63), dict(ld_dx=63), dict(ld_dw_gate=63), dict(ld_dw_up=65),
                                    dict(ld_dw_down=95), dict(dy=1), dict(dw_gate=1)])
def test_ffn_gradient_refusals(change):
    assert _sizes(_ffn(), _grads(**change))[0] == B.ERR_ARG
    assert B.lib().chm_ffn_backward(_ffn(), _grads(**change), None, 0, None) == B.ERR_ARG


def test_null_pointers():
    L = B.lib()
    assert L.chm_ffn_sizes(None, None, None, None, None) == B.ERR_ARG
    assert L.chm_ffn_forward(None, None, 64, None, 0, None) == B.ERR_ARG
    assert L.chm_ffn_forward(_ffn(), None, 64, None, 0, None) == B.ERR_ARG
    assert L.chm_ffn_backward(_ffn(), None, None, 0, None) == B.ERR_ARG
    assert L.chm_embedding_lookup(1, 64, None, 5, None, 8, 10, 8, 1.0, None, 8, None) == B.ERR_ARG
    assert L.chm_embedding_gradient(1, 1, 64, None, 5, None, 8, 10, 8, 1.0, None, 8, 0, None, 0, None) == B.ERR_ARG
    assert L.chm_gradient_sumsq(None, None, None) == B.ERR_ARG
    assert L.chm_clip_gradients(None, 1.0, None, None, None) == B.ERR_ARG
    assert L.chm_load_gradients(None, 1, None) == B.ERR_ARG
    L.chm_free_gradients(None)
    assert L.chm_ffn_forward(_ffn(T=0), None, 64, None, 0, None) == B.OK               # nothing to do


def test_embedding_sizes_and_refusals():
    L, n = B.lib(), C.c_uint64()
    assert L.chm_embedding_gradient_scratch(512, 1000, 64, n) == B.OK and n.value == 0
    assert L.chm_embedding_gradient_scratch(513, 1000, 64, n) == B.OK and n.value >= 513 * 16 + 1000
    for args in ((-1, 10, 8), (5, -1, 8), (5, 10, 0), (1 << 31, 10, 8), (5, 1 << 31, 8)):
        assert L.chm_embedding_gradient_scratch(*args, n) == B.ERR_ARG
    assert L.chm_embedding_gradient_scratch(5, 5, 5, None) == B.ERR_ARG

    def lookup(dtype=1, bits=64, n=0, ld=8, rows=10, width=8, ld_out=8):
        return L.chm_embedding_lookup(dtype, bits, None, n, None, ld, rows, width, 1.0, None, ld_out, None)

    assert lookup() == B.OK
    for change in (dict(dtype=3), dict(bits=16), dict(n=-1), dict(ld=7), dict(rows=-1), dict(width=0), dict(ld_out=7)):
        assert lookup(**change) == B.ERR_ARG, change


def test_loading_gradients_refuses_before_the_device():
    h = C.c_void_p()
    for bad in (B.Gradient(None, None, 5, 0), B.Gradient(2, None, 5, 0), B.Gradient(4, 2, 5, 0), B.Gradient(4, None, -1, 0), B.Gradient(4, None, 5, 3)):
        assert B.lib().chm_load_gradients(bad, 1, h) == B.ERR_ARG and not h.value
    assert B.lib().chm_load_gradients(None, -1, h) == B.ERR_ARG


def test_tensors_that_are_not_on_the_gpu_are_refused():
    x, w, d = torch.zeros(2, 8).bfloat16(), torch.zeros(16, 8).bfloat16(), torch.zeros(8, 16).bfloat16()
    for call in (lambda: ops.ffn_forward(x, w, w, d), lambda: ops.embedding_lookup(torch.zeros(3, dtype=torch.int64), w),
                 lambda: ops.embedding_gradient(x, torch.zeros(2, dtype=torch.int64), 4), lambda: ops.ffn_forward(None, w, w, d)):
        with pytest.raises(B.ChmError) as e:
            call()
        assert e.value.code == B.ERR_ARG


def test_gradients_that_are_no_tensors_are_refused():
    """a parameter's missing gradient among them"""
    for bad in ([None], [3.0], [None, torch.zeros(3)], [torch.zeros(3), None]):
        with pytest.raises(B.ChmError) as e:
            ops.Gradients(bad)
        assert e.value.code == B.ERR_ARG, bad


def test_shapes_of_the_gpu_tests_reach_every_kernel_of_the_block():
    from tests.test_operators import FFN_KERNELS
    reached = set()
    for T, D, F in FFN_KERNELS:
        k = B.FfnKernels()
        assert B.lib().chm_ffn_selection(_ffn(T, D, F, ld_x=D, ld_gate=D, ld_up=D, ld_down=F), _grads(T, D, F), k) == B.OK
        reached |= {("tile", p, k.tile[p], k.splits[p] > 1) for p in range(4) if k.tile[p] >= 0}
        reached |= {("few", p, k.few, k.few_slices[p], k.few_ends[p]) for p in range(2) if k.few}
    products = {0: (4, False), 1: (4, True), 2: (4, False), 3: (3, True)}              # kinds of tile, whether sums may be split
    want = {("tile", p, t, s) for p, (tiles, split) in products.items() for t in range(tiles) for s in {False, split}}
    want |= {("few", p, blocks, slices, ends) for p in (0, 1) for blocks, slices in ((1, 1), (1, 2), (1, 4), (2, 1), (3, 1)) for ends in (0, 1)}
    assert reached == want


def test_ffn_selection_refuses_what_the_calls_refuse():
    L, k = B.lib(), B.FfnKernels()
    assert L.chm_ffn_selection(_ffn(), None, k) == B.OK and list(k.tile[2:]) == [-1, -1]
    assert L.chm_ffn_selection(None, None, k) == L.chm_ffn_selection(_ffn(), None, None) == L.chm_ffn_selection(_ffn(dtype=0), None, k) == B.ERR_ARG
    assert L.chm_ffn_selection(_ffn(), _grads(grad_dtype=2), k) == L.chm_ffn_selection(_ffn((1 << 31) - 1, 8, 8), None, k) == B.ERR_ARG


def test_structure_of_the_selection_matches_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "chm_measure.h"\nint main(void) { printf("%zu", sizeof(chm_ffn_kernels));' +
                   "".join('printf(" %%zu", offsetof(chm_ffn_kernels, %s));' % f for f, _ in B.FfnKernels._fields_) + " return 0; }")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), "-o", str(tmp_path / "layout"), str(src)], check=True)
    out = [int(v) for v in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.split()]
    assert out == [C.sizeof(B.FfnKernels)] + [getattr(B.FfnKernels, f).offset for f, _ in B.FfnKernels._fields_]


def test_structures_match_the_header(tmp_path):
    """sizes and field offsets of the binding's structures against what a C compiler makes of include/chm_operators.h"""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"chm_ffn": B.Ffn, "chm_ffn_gradients": B.FfnGradients, "chm_gradient": B.Gradient}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "chm_operators.h"', 'int main(void) {']
    for cname, cls in structs.items():
        lines.append('  printf("%s %%zu\\n", sizeof(%s));' % (cname, cname))
        lines += ['  printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (cname, f, cname, f) for f, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ['  return 0;', '}']))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), "-o", str(tmp_path / "layout"), str(src)], check=True)
    out = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout
    want = dict(line.split() for line in out.splitlines())
    for cname, cls in structs.items():
        assert C.sizeof(cls) == int(want[cname]), cname
        for field, _ in cls._fields_:
            assert getattr(cls, field).offset == int(want["%s.%s" % (cname, field)]), (cname, field)
