"""A round between a program's tensors on the GPU, used as a training step would: gradients of many tensors of mixed types,
clipped and gathered, through the round (against the same round on vectors made with torch), the residual of error feedback over
rounds, and the average into weights by an Adam step or into tensors; on one GPU and through the data-parallel path."""
import gc
import math
import os
import socket

import pytest
import torch

import tensor_lists as T
from tensor_lists import U

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def nothing_left_behind():
    """What a caught exception's frames hold (tensors) goes with the test, not in the middle of a later one."""
    yield
    gc.collect()


SIZES = [40_000, 1, 333, 64, 7_001, 20_000, 5]


def context(n=3, k=12, in_dtype=0):
    from paper_2302_08545_b200 import thc, workloads as W
    return thc.Context(bits=4, granularity=30, table=W.TABLES[(4, 30)], t_p=W.T_P["1/32"], log2_block=k, seed=W.THC_SEED, workers=n, in_dtype=in_dtype)


@pytest.mark.parametrize("types", [["f32"], ["bf16", "f32", "f16"]])
@pytest.mark.parametrize("flat", ["f32", "bf16"])
def test_a_round_of_tensors_is_the_round_of_their_vectors(types, flat):
    from paper_2302_08545_b200 import runner
    ctx = context(in_dtype=1 if flat == "bf16" else 0)
    grads = T.make(SIZES, types, 3, seed=1)
    tr = runner.TensorRound(ctx, grads)
    plain = runner.Round(ctx, 3, tr.grads.d, flat)
    for most in (math.inf, 50.0):
        out = tr.run(4, max_norm=most).clone()
        for x, w in zip(plain.grads, grads):
            x.zero_()
            c = T.factor(T.norm(w), most)
            for v, g in zip(tr.grads.views(x), w):
                v.copy_(g.double() * c)
        for x, y in zip(tr.round.grads, plain.grads):      # one rounding more than from 64 bits, and the factor's two and a half
            T.within(x, y.double(), y.double().abs() * ((2.0 ** -8 if flat == "bf16" else 0.0) * 2 + 4.5 * U) + 2.0 ** -149)
        for x, y in zip(tr.round.grads, plain.grads):
            y.copy_(x)
        plain.run(4, fused=True)
        assert torch.equal(plain.out, out) and torch.equal(plain.scales, tr.round.scales)
    ref = torch.tensor([T.norm(w) for w in grads], dtype=torch.float64)
    T.within(tr.norms.cpu(), ref, ref * 2.6 * U)
    assert ctx.status() == 0


def test_error_feedback_over_rounds():
    from paper_2302_08545_b200 import runner
    ctx = context()
    grads = T.make(SIZES, ["f32", "bf16"], 3, seed=2)
    tr = runner.TensorRound(ctx, grads, error_feedback=True)
    plain = runner.Round(ctx, 3, tr.grads.d)
    ef = [torch.zeros(tr.grads.d, device="cuda") for _ in range(3)]
    for rnd in range(3):
        for x, w, e in zip(plain.grads, grads, ef):
            x.zero_()
            for v, g in zip(tr.grads.views(x), w):
                v.copy_(g)
            x.add_(e)                                      # without clipping c = 1: one rounding either way
        plain.run(rnd, fused=True)
        ctx.error_feedback(plain.grads, plain.packed, plain.d, rnd, plain.scales, ef, plain.workspace)
        assert torch.equal(tr.run(rnd), plain.out)
        assert all(torch.equal(a, b) for a, b in zip(tr.ef, ef))


def test_training_step_by_step():
    """Three steps of a least-squares model from its tensors' gradients: every weight is the formula's, from the average that the
    round gave."""
    from paper_2302_08545_b200 import runner, thc
    ctx = context(n=2)
    sizes, types = [600, 30, 7], ["bf16", "bf16", "f32"]
    weights = T.make(sizes, types, 1, seed=3, scale=0.1)
    grads = T.make(sizes, types, 2, seed=4)
    tr = runner.TensorRound(ctx, grads, error_feedback=True)
    wl = thc.Tensors(ctx, weights)
    d = wl.d
    assert d == tr.grads.d and wl.offsets == tr.grads.offsets
    master, m, v = (torch.zeros(d, device="cuda") for _ in range(3))
    for x, w in zip(wl.views(master), weights[0]):
        x.copy_(w)
    lr, step = torch.full((1,), 0.05, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    em, ev, ew = (x.double() for x in (m, v, master))
    for t in range(1, 4):
        for wk in range(2):                                # gradients of |w - 1|^2 / 2 with a worker's own noise
            for g, w in zip(grads[wk], weights[0]):
                g.copy_(w.double() - 1.0 + 0.01 * torch.randn(w.shape, device="cuda", dtype=torch.float64))
        out = tr.run(t, max_norm=10.0)
        tr.adamw(wl, lr, step, m, v, master=master, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.01, max_norm=1.0)
        views = [wl.views(out.double())]
        c = T.factor(T.norm(views[0]), 1.0)
        for i, g in enumerate(views[0]):
            pm, pv, pw = (wl.views(x)[i] for x in (em, ev, ew))
            pm.mul_(0.9).add_(0.1 * c * g)
            pv.mul_(0.99).add_(0.01 * (c * g) ** 2)
            pw.copy_(pw * (1 - float(lr) * 0.01) - float(lr) * (pm / (1 - 0.9 ** t)) / (torch.sqrt(pv / (1 - 0.99 ** t)) + 1e-6))
        # per step: the bounds of one step (at most 10 u of the step, which is at most lr / sqrt(1 - b2) = 10 lr, and 3 u |w|), and
        # what the moments were off before, which moves the quotient by no more; three steps
        assert float((master.double() - ew)[: 600].abs().max()) <= t * U * (40 * 10 * 0.05 + 4)
        for x, y in zip(weights[0], wl.views(master)):
            assert torch.equal(x, y.to(x.dtype))
    assert int(step) == 3 and ctx.status() == 0
    back = thc.Tensors(ctx, T.make(sizes, ["f16", "bf16", "f32"], 1))
    tr.scatter(back, max_norm=0.5)
    for x, g in zip(back.tensors[0], back.views(tr.round.out)):
        exact = g.double() * T.factor(T.norm(back.views(tr.round.out)), 0.5)
        rel, least = T.half_step(x.dtype)
        T.within(x, exact, exact.abs() * (2.1 * U + (rel if x.dtype != torch.float32 else 0)) + least + 2.0 ** -149)


def test_one_rank_of_the_data_parallel_round():
    import torch.distributed as dist
    from paper_2302_08545_b200 import runner, thc
    from paper_2302_08545_b200.data_parallel import CudaOps, DataParallelRound
    dev = torch.device("cuda", 0)
    torch.cuda.set_device(dev)
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    os.environ["MASTER_ADDR"], os.environ["MASTER_PORT"] = "127.0.0.1", str(port)
    dist.init_process_group("nccl", rank=0, world_size=1, device_id=dev)
    try:
        ctx = context(n=1)
        grads = T.make(SIZES, ["bf16", "f32"], 1, seed=5)
        lst = thc.Tensors(ctx, grads)
        ops = CudaOps(ctx, lst.d, dev)
        dp = DataParallelRound(ops, lst.d, 12, 4, ctx.sizes(lst.d, 1).acc_bits)
        tr = runner.TensorRound(ctx, grads, error_feedback=True)
        ef = torch.zeros(lst.d, device=dev)
        for rnd in range(2):
            expected = tr.run(rnd, max_norm=3.0).clone()
            out, _, _, _ = dp.step_tensors(lst, rnd, max_norm=3.0, ef=ef)
            assert torch.equal(out, expected) and torch.equal(ef, tr.ef[0]) and torch.equal(ops.norm, tr.norms)
        weights = T.make(SIZES, ["f32"], 2, seed=6)
        state = [[torch.zeros(lst.d, device=dev) for _ in range(2)] for _ in range(2)]
        lr, step = torch.full((1,), 0.1, device=dev), torch.zeros(2, dtype=torch.int64, device=dev)
        for x, y in zip(*weights):
            y.copy_(x)
        ops.adamw(out, thc.Tensors(ctx, weights[:1]), lr, step[:1], *state[0], max_norm=1.0)
        tr.round.out.copy_(out)
        tr.adamw(thc.Tensors(ctx, weights[1:]), lr, step[1:], *state[1], max_norm=1.0)
        assert all(torch.equal(x, y) for x, y in zip(*weights)) and step.tolist() == [1, 1]
        ops.scatter(out, lst, max_norm=1.0)
        norm = T.norm(lst.views(out))
        T.within(ops.average_norm.cpu(), torch.tensor([norm], dtype=torch.float64), torch.tensor([norm * 1.1 * U], dtype=torch.float64))
        for x, g in zip(grads[0], lst.views(out)):
            exact = g.double() * T.factor(norm, 1.0)
            T.within(x, exact, exact.abs() * (2.1 * U + (2.0 ** -8 if x.dtype == torch.bfloat16 else 0)) + 2.0 ** -149)
    finally:
        dist.destroy_process_group()


def test_a_captured_training_step():
    """Gather, round and Adam step as one CUDA graph, replayed: the same as the calls."""
    from paper_2302_08545_b200 import runner, thc
    ctx = context(n=2, k=10)
    grads = T.make(SIZES, ["bf16", "f32"], 2, seed=7)
    weights = T.make(SIZES, ["bf16"], 1, seed=8)
    tr = runner.TensorRound(ctx, grads, error_feedback=True)
    wl = thc.Tensors(ctx, weights)
    state = [torch.zeros(wl.d, device="cuda") for _ in range(3)]
    lr, step = torch.full((1,), 0.1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")

    def call():
        tr.run(1, max_norm=1.0)
        tr.adamw(wl, lr, step, state[0], state[1], master=state[2], max_norm=0.5, weight_decay=0.1)
    every = [*state, *weights[0], *tr.ef, step]
    start = [x.clone() for x in every]
    for _ in range(3):
        call()
    torch.cuda.synchronize()
    expected = [x.clone() for x in every]
    for x, y in zip(every, start):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(every, expected)) and int(step) == 3
