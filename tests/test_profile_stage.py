"""A stage's training step on the operators, end to end: its gradients and norm against the formulas in 64 bits, and a scenario of measured
tables against the oracle."""
import numpy as np
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


def _reference(stage, micro, dys):
    """gradients of the step in 64 bits by autograd"""
    table = stage.table.double().requires_grad_(True)
    blocks = [[w.double().requires_grad_(True) for w in b] for b in stage.blocks]
    loss = 0
    for tokens, dy in zip(micro, dys):
        x = table[tokens] * stage.scale
        for wg, wu, wd in blocks:
            x = (torch.nn.functional.silu(x @ wg.T) * (x @ wu.T)) @ wd.T
        loss = loss + (x * dy.double()).sum()
    loss.backward()
    return [w.grad for b in blocks for w in b] + [table.grad]


@pytest.mark.parametrize("tokens,ahead", [(7, 0), (150, 1), (150, 5)])
def test_step_against_autograd(stage_module, tokens, ahead):
    T, D, F, V, M = tokens, 72, 136, 50, 3
    stage = stage_module.Stage(2, D, F, V, dtype=torch.float16, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    micro = [torch.randint(V, (T,), generator=g, device="cuda") for _ in range(M)]
    dys = [(torch.randn(T, D, generator=g, device="cuda") * 0.1).half() for _ in range(M)]
    want = _reference(stage, micro, dys)
    norm, _ = stage.step(micro, lambda k, y: dys[k], max_norm=1e9, ahead=ahead)
    got = [t for b in stage.grads for t in b] + [stage.table_grad]
    # between the inputs and a gradient lie at most a dozen roundings to 11 bits of independent values, each of a relative standard
    # deviation of 2^-11 / sqrt(3): six standard deviations of a gradient's error as a whole
    tol = 6 * 12 ** 0.5 * 2.0 ** -11 / 3 ** 0.5
    for a, b in zip(got, want):
        assert float((a.double() - b).norm() / b.norm()) <= tol
    total = float(sum((b ** 2).sum() for b in want)) ** 0.5
    assert abs(float(norm) - total) <= tol * total
    again = [t.clone() for t in got]
    norm2, _ = stage.step(micro, lambda k, y: dys[k], max_norm=total / 2, ahead=ahead)      # the same step, clipped
    assert float(norm2) == float(norm)
    for a, b in zip(got, again):
        assert torch.allclose(a, b * (total / 2 / float(norm)), rtol=1e-3, atol=0)


def test_a_step_of_no_micro_batches_has_no_gradients(stage_module):
    stage = stage_module.Stage(1, 64, 72, 30)
    tokens = torch.arange(20, device="cuda")
    assert float(stage.step([tokens], lambda k, y: y, max_norm=1.0)[0]) > 0
    norm, dx = stage.step([], lambda k, y: y, max_norm=1.0)
    assert float(norm) == 0 and dx == [] and not any(bool(t.any()) for b in stage.grads for t in b) and not bool(stage.table_grad.any())


def test_stage_without_embedding_returns_the_gradients_of_its_inputs(stage_module):
    stage = stage_module.Stage(1, 64, 72, dtype=torch.float16)
    x = [torch.randn(20, 64, device="cuda").half() for _ in range(2)]
    _, dx = stage.step(x, lambda k, y: y, max_norm=1.0)
    assert len(dx) == 2 and dx[0].shape == (20, 64) and bool(torch.isfinite(dx[1]).all())


def test_scenario_of_measured_tables(stage_module):
    from oracle import oracle as O
    from paper_2508_21613_amd import binding as B
    stage = stage_module.Stage(1, 256, 512, 1000)
    tables = stage_module.measure(stage, 64, repeats=3)
    assert all(len(v) == 2 and min(v) >= 0 for v in tables.values()) and min(tables["fwd_us"] + tables["bwd_us"]) >= 1
    sc = stage_module.scenario(tables, 12, 3, 2, 4, [1], 150, 10000)
    assert sc["fwd_us"][0] == sum(tables["fwd_us"]) and sc["fwd_us"].dtype == np.int32
    rc, best = B.Scenario(sc).search_best()
    assert (rc, best) == O.Scenario(sc).search(7)


def test_times_are_those_of_the_gpu(stage_module, monkeypatch):
    """a host that takes milliseconds to make a layer's calls adds nothing to its times"""
    import time
    stage = stage_module.Stage(1, 128, 256, 500)

    def late(call):
        def f(*args, **kw):
            time.sleep(0.003)
            return call(*args, **kw)
        return f

    monkeypatch.setattr(stage, "forward_layer", late(stage.forward_layer))
    monkeypatch.setattr(stage, "backward_layer", late(stage.backward_layer))
    tables = stage_module.measure(stage, 20, repeats=3)
    assert max(tables["fwd_us"] + tables["bwd_us"]) < 1000, tables


def test_command(stage_module, capsys):
    assert stage_module.main(["--layers", "8", "--width", "128", "--features", "256", "--vocabulary", "500", "--tokens", "50", "--pp", "4"]) == 0
    assert "best plan after the loss of [3]" in capsys.readouterr().out
