"""A training step of embedding and feed-forward blocks on this package's operators, and a scenario's tables measured from it.

    python -m paper_2508_21613_amd.profile_stage --layers 32 --width 4096 --features 11008 --vocabulary 32000 --tokens 4096 \\
        --pp 4 --dp 2 --micro-batches 8 --failed 3

A scenario wants the forward and backward time and the memory of every layer, which the paper's profiler collects at run time (System
Design, workflow step 1): a job's tables come from the job.  `Stage` runs the part of such a step that this package has operators for: the
embedding of the first stage and gated feed-forward blocks (no attention, norms, output head or optimizer), forward and backward over the
micro-batches of a step in 1F1B order, gradients added up in float32 and clipped at the end.  `measure` times every layer on the GPU with
events (the clipping is the step's, and in no table), `scenario` makes a scenario of the tables, and the command searches it for the best plan
after the given failures.
"""
import argparse
import collections
import statistics

import numpy as np
import torch

from . import binding, operators, synth

MIB = 1 << 20


class Stage:
    """`layers` feed-forward blocks, behind an embedding if `vocabulary` is given.  Weights are random; gradients are float32."""

    def __init__(self, layers, width, features, vocabulary=0, dtype=torch.bfloat16, activation="silu", seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(rows, cols):
            return torch.empty((rows, cols), dtype=dtype, device=device).normal_(0.0, cols ** -0.5, generator=g)

        self.width, self.activation = width, activation
        self.scale = width ** 0.5
        self.table = weight(vocabulary, width) if vocabulary else None
        self.blocks = [(weight(features, width), weight(features, width), weight(width, features)) for _ in range(layers)]
        self.grads = [tuple(torch.zeros(w.shape, device=device) for w in block) for block in self.blocks]
        self.table_grad = torch.zeros(self.table.shape, device=device) if vocabulary else None
        flat = [t for block in self.grads for t in block] + ([self.table_grad] if vocabulary else [])
        self.clipper = operators.Gradients(flat)

    # one layer at a time: layer -1 is the embedding
    def forward_layer(self, i, x):
        """(result, what the backward pass needs)"""
        if i < 0:
            return operators.embedding_lookup(x, self.table, self.scale), x
        y, saved = operators.ffn_forward(x, *self.blocks[i], activation=self.activation, save=True)
        return y, (x, saved)

    def backward_layer(self, i, dy, kept, first):
        """the gradient of the layer's input (None for the embedding); `first`: of the step's micro-batches, whose gradients are written"""
        if i < 0:
            operators.embedding_gradient(dy, kept, scale=self.scale, out=self.table_grad, accumulate=not first)
            return None
        x, saved = kept
        return operators.ffn_backward(dy, x, *self.blocks[i], saved, activation=self.activation, grads=self.grads[i], accumulate=not first)[0]

    @property
    def layers(self):
        return list(range(-1 if self.table is not None else 0, len(self.blocks)))

    def step(self, inputs, gradient_of, max_norm, ahead=0, sumsq=None):
        """One training step: forward and backward of every micro-batch of `inputs` (tokens, or [tokens, width] from the stage before),
        at most `ahead` + 1 of them in flight as in 1F1B with `ahead` stages behind this one.  gradient_of(k, y): the gradient
        with respect to the result of micro-batch k.  Returns the gradient norm (`sumsq`: of all stages) and, for a stage without an
        embedding, the gradients with respect to the inputs."""
        flying, to_inputs, k = collections.deque(), [], None

        def backward():
            k, y, kept = flying.popleft()
            d = gradient_of(k, y)
            for i in reversed(self.layers):
                d = self.backward_layer(i, d, kept.pop(), first=k == 0)
            to_inputs.append(d)

        for k, x in enumerate(inputs):
            kept = []
            for i in self.layers:
                x, needed = self.forward_layer(i, x)
                kept.append(needed)
            flying.append((k, x, kept))
            if len(flying) > ahead:
                backward()
        while flying:
            backward()
        if k is None:                                                      # the last step's gradients are not this one's
            for t in [t for block in self.grads for t in block] + ([] if self.table is None else [self.table_grad]):
                t.zero_()
        return self.clipper.clip(max_norm, sumsq=sumsq), to_inputs


class _Queued:
    """Times of calls on the GPU alone: fills of a large buffer keep it busy until the calls between two marks have all been made, more of them
    as long as it came to the first mark before that.  The calls find their operands out of the caches, as in a step."""

    def __init__(self, device):
        self.buffer = torch.empty(1 << 26, device=device)                  # some 40 us a fill
        self.fills, self.most = 4, 4096

    def __call__(self, *calls):
        """ms of each call, made in turn"""
        while True:
            marks = [torch.cuda.Event(enable_timing=True) for _ in range(len(calls) + 1)]
            for _ in range(self.fills):
                self.buffer.zero_()
            marks[0].record()
            for call, mark in zip(calls, marks[1:]):
                call()
                mark.record()
            early = marks[0].query()
            marks[-1].synchronize()
            if not early or self.fills >= self.most:
                return [a.elapsed_time(b) for a, b in zip(marks, marks[1:])]
            self.fills *= 2


def measure(stage, tokens, repeats=10, optimizer_bytes=12, seed=1):
    """Tables of the stage's layers (the embedding first, if it has one) for micro-batches of `tokens` tokens: forward and backward time
    in us (medians on the GPU, at least 1), MiB of weights, float32 gradients and `optimizer_bytes` per weight, MiB kept per micro-batch in flight."""
    dev = stage.blocks[0][0].device if stage.blocks else stage.table.device
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    some = stage.blocks[0][0] if stage.blocks else stage.table
    fwd, bwd, mem, act = [], [], [], []
    timed = _Queued(dev)
    for i in stage.layers:
        if i < 0:
            x = torch.randint(stage.table.shape[0], (tokens,), generator=g, device=dev)
            weights = [stage.table]
        else:
            x = torch.empty((tokens, stage.width), dtype=some.dtype, device=dev).normal_(0.0, 1.0, generator=g)
            weights = stage.blocks[i]
        dy = torch.empty((tokens, stage.width), dtype=some.dtype, device=dev).normal_(0.0, 0.05, generator=g)
        kept = None

        def forward():
            nonlocal kept
            kept = stage.forward_layer(i, x)[1]

        times = [timed(forward, lambda: stage.backward_layer(i, dy, kept, first=False)) for _ in range(repeats + 2)]
        times = [statistics.median(t) for t in zip(*times[2:])]            # the first ones load the kernels
        fwd.append(max(1, round(times[0] * 1e3)))
        bwd.append(max(1, round(times[1] * 1e3)))
        n = sum(w.numel() for w in weights)
        mem.append(-(-n * (some.element_size() + 4 + optimizer_bytes) // MIB))
        held = [kept] if torch.is_tensor(kept) else kept
        act.append(-(-sum(t.numel() * t.element_size() for t in held) // MIB))
    return {"fwd_us": fwd, "bwd_us": bwd, "mem_mib": mem, "act_mib": act}


def scenario(tables, layers, pp, dp, micro_batches, failed, comm_us, mem_cap_mib, **kw):
    """The scenario of a model of `layers` equal blocks behind an embedding: `tables` (measure) of a stage with an embedding and one
    block.  The embedding's times, weights and kept tokens are added to the first block's: it runs on the same node."""
    def spread(name):
        first, block = tables[name]
        a = np.full(layers, block, dtype=np.int32)
        a[0] += first
        return a

    return synth.scenario(layers, pp, dp, micro_batches, spread("fwd_us"), spread("bwd_us"), spread("mem_mib"), failed, comm_us, mem_cap_mib,
                          act_mib=spread("act_mib"), **kw)


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value, text in (("layers", 32, "feed-forward blocks of the model"), ("width", 4096, "elements of a token"),
                              ("features", 11008, "features of a block"), ("vocabulary", 32000, "rows of the embedding"),
                              ("tokens", 4096, "tokens of a micro-batch"), ("pp", 4, "stages"), ("dp", 2, "pipelines"),
                              ("micro-batches", 8, "micro-batches of a pipeline"), ("comm-us", 150, "time of a stage boundary"),
                              ("mem-cap-mib", 288 * 1024 * 9 // 10, "memory of a node")):
        p.add_argument("--" + name, type=int, default=value, help="%s (%d)" % (text, value))
    p.add_argument("--failed", type=int, nargs="+", default=[3], help="nodes that have failed, pipeline x stages + stage (3)")
    a = p.parse_args(argv)
    stage = Stage(1, a.width, a.features, a.vocabulary)
    micro = [torch.randint(a.vocabulary, (a.tokens,), device="cuda") for _ in range(2)]
    norm, _ = stage.step(micro, lambda k, y: y * 1e-3, max_norm=1.0, ahead=1)
    tables = measure(stage, a.tokens)
    print("one step of an embedding and a block: gradient norm %.4g" % float(norm))
    for name, values in tables.items():
        print("%-8s embedding %6d   block %6d" % (name, *values))
    g = binding.Scenario(scenario(tables, a.layers, a.pp, a.dp, a.micro_batches, a.failed, a.comm_us, a.mem_cap_mib))
    rc, best = g.search_best()
    if rc != binding.OK:
        print("no plan:", binding.strerror(rc))
        return 1
    strategy = ("redundant computation", "re-partition", "data rerouting")[best["strategy"]]
    print("best plan after the loss of %s: %s, %d stages, cuts %s, step %d us, transition %d us"
          % (a.failed, strategy, best["stages"], best["cuts"], best["t_step_us"], best["t_trans_us"]))
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
