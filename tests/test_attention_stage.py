"""What lies between an attention's projections as a stage runs it: rotary positions, attention, their gradients in one buffer, against autograd in 64
bits; and a scenario of the times measured of it, against the oracle."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def stage_module():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_21613_amd import binding, profile_stage
    binding.lib()
    return profile_stage


def _reference(a, qkv, pos, documents, prefix, dy, slopes, cap, axes):
    """(y, gradient of qkv) in 64 bits by autograd"""
    x = qkv.double().requires_grad_(True)
    T, H, Hk, d = len(x), a.heads, a.kv_heads, a.head_dim
    P = len(axes)
    freq = torch.tensor([10000.0 ** (-i / P) for i in range(P)], dtype=torch.float64, device="cuda")
    angle = (pos.double()[torch.tensor(axes, device="cuda")].T * freq)[:, None]
    both = x[:, :H + Hk]
    one, two = both[..., :P], both[..., P:2 * P]
    both = torch.cat([one * angle.cos() - two * angle.sin(), one * angle.sin() + two * angle.cos(), both[..., 2 * P:]], dim=-1)
    q, k, v = both[:, :H], both[:, H:].repeat_interleave(H // Hk, 1), x[:, H + Hk:].repeat_interleave(H // Hk, 1)
    s = torch.stack([q[:, h] @ k[:, h].T for h in range(H)]) * d ** -0.5
    if cap:
        s = cap * torch.tanh(s / cap)
    i = torch.arange(T, device="cuda")
    if slopes is not None:
        s = s - slopes.double()[:, None, None] * (i[:, None] - i).abs()
    see = i <= i[:, None]
    if prefix is not None:
        see = see | prefix
    if documents is not None:
        see = see & (documents[:, None] == documents) & (documents >= 0)
    some = see.any(1)
    p = torch.softmax(s.masked_fill(~(see | ~some[:, None]), -torch.inf), -1) * some[:, None]
    y = torch.stack([p[h] @ v[:, h] for h in range(H)], dim=1)
    (y * dy.double()).sum().backward()
    return y.detach(), x.grad


@pytest.mark.parametrize("tokens,heads,kv_heads,dim,sections,cap,slopes,masks", [
    (7, 2, 2, 64, None, 0.0, False, False), (150, 6, 2, 64, [8, 12, 12], 0.0, False, True), (300, 4, 1, 128, None, 10.0, False, False),
    (200, 4, 4, 80, [10, 30], 5.0, True, True)])
def test_forward_and_backward_against_autograd(stage_module, tokens, heads, kv_heads, dim, sections, cap, slopes, masks):
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    slope = torch.exp2(-torch.arange(1.0, heads + 1, device="cuda")) if slopes else None
    a = stage_module.Attention(heads, kv_heads, dim, sections=sections, cap=cap, slopes=slope)
    axes = [0] * (dim // 2) if sections is None else [i for i, n in enumerate(sections) for _ in range(n)]
    qkv = torch.randn((tokens, heads + 2 * kv_heads, dim), generator=g, device="cuda").half()
    dy = (torch.randn((tokens, heads, dim), generator=g, device="cuda") * 0.2).half()
    pos = torch.randint(0, 3000, (max(axes) + 1, tokens), generator=g, device="cuda")
    documents = prefix = None
    if masks:
        documents = torch.arange(tokens, device="cuda") // 60
        documents[-20:] = -1
        prefix = torch.arange(tokens, device="cuda") % 60 < 25
    want_y, want = _reference(a, qkv, pos, documents, prefix, dy, slope, cap, axes)
    y, kept = a.forward(qkv, pos, documents, prefix)
    grad = a.backward(dy, kept)
    assert grad.shape == qkv.shape
    # between the inputs and a gradient lie at most a dozen roundings to 11 bits of independent values (turned queries and keys, weights, ds, results),
    # each of a relative standard deviation of 2^-11 / sqrt(3), those of the turned ones amplified by the scores' size: six standard deviations as a whole
    tol = 6 * 12 ** 0.5 * 2.0 ** -11 / 3 ** 0.5
    assert float((y.double() - want_y).norm() / want_y.norm()) <= tol
    H, K = heads, heads + kv_heads
    for part in (slice(0, H), slice(H, K), slice(K, None)):
        assert float((grad[:, part].double() - want[:, part]).norm() / want[:, part].norm()) <= tol
    again = a.backward(dy, a.forward(qkv, pos, documents, prefix)[1])
    assert torch.equal(grad, again)


def test_scenario_with_attention(stage_module):
    from oracle import oracle as O
    from paper_2508_21613_amd import binding as B
    stage = stage_module.Stage(1, 256, 512, 1000)
    tables = stage_module.measure(stage, 64, repeats=3)
    extra = stage_module.measure_attention(stage_module.Attention(4, 2, 64, sections=[10, 11, 11]), 64, repeats=3)
    assert extra["fwd_us"] >= 1 and extra["bwd_us"] >= 1 and extra["act_mib"] >= 1
    plain = stage_module.scenario(tables, 12, 3, 2, 4, [1], 150, 10000)
    sc = stage_module.scenario(tables, 12, 3, 2, 4, [1], 150, 10000, attention=extra)
    for name, add in extra.items():
        assert (sc[name] - plain[name] == add).all()
    assert (sc["mem_mib"] == plain["mem_mib"]).all()
    rc, best = B.Scenario(sc).search_best()
    assert (rc, best) == O.Scenario(sc).search(7)


def test_command(stage_module, capsys):
    assert stage_module.main(["--layers", "8", "--width", "128", "--features", "256", "--vocabulary", "500", "--tokens", "50", "--pp", "4", "--heads", "4", "--kv-heads", "2",
                              "--documents", "3"]) == 0
    out = capsys.readouterr().out
    assert "attention's part between its projections" in out and "best plan after the loss of [3]" in out
