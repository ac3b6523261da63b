"""Rounds with a gradient that is not finite, on the GPU: what thc_void_round writes and leaves alone, and training steps through
runner.TensorRound with such a round among them, which go on as if it had not been."""
import gc
import math

import pytest
import torch

import tensor_lists as T

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def nothing_left_behind():
    yield
    gc.collect()


def context(n=3, k=12, in_dtype=0):
    from paper_2302_08545_b200 import thc, workloads as W
    return thc.Context(bits=4, granularity=30, table=W.TABLES[(4, 30)], t_p=W.T_P["1/32"], log2_block=k, seed=W.THC_SEED, workers=n, in_dtype=in_dtype)


@pytest.mark.parametrize("size", [1, 300, 70_001, 3_000_001])
@pytest.mark.parametrize("n,k", [(1, 6), (3, 12), (64, 8)])
@pytest.mark.parametrize("residuals", [False, True])
def test_what_is_written(size, n, k, residuals):
    from paper_2302_08545_b200 import thc
    if size > 1_000_000 and n > 3:
        pytest.skip("one large case of each kind")
    ctx = context(n, k)
    lst = thc.Tensors(ctx, [[torch.zeros(size, device="cuda")] for _ in range(n)])
    scales_n = ctx.sizes(lst.d, 1).scales_count
    room = [torch.randn(lst.d + 64, device="cuda") for _ in range(1 + 2 * n)]
    (out, *rest), scales = [x[: lst.d] for x in room], torch.rand(scales_n + 64, device="cuda")
    grads, ef = (rest[:n], rest[n:]) if residuals else (None, None)
    norms = torch.rand(n, device="cuda")
    every = [*room, scales, norms]
    old = [x.clone() for x in every]
    ctx.void_round(lst, math.inf, norms, scales[:scales_n], out, grads, ef)
    assert all(torch.equal(x, y) for x, y in zip(every, old)) and ctx.status() == 0
    for i, value in {0: math.nan, n - 1: math.inf}.items():
        for x, y in zip(every, old):
            x.copy_(y)
        norms[i] = value
        ctx.void_round(lst, math.inf, norms, scales[:scales_n], out, grads, ef)
        assert ctx.status() == thc.STATUS_NONFINITE
        assert bool(torch.isnan(out).all()) and not bool(scales[:scales_n].any())
        assert torch.equal(scales[scales_n:], old[-2][scales_n:])
        for r, (x, y) in enumerate(zip(room, old)):
            assert torch.equal(x[lst.d:], y[lst.d:])
            if 1 <= r <= n and residuals:
                assert torch.equal(x[: lst.d], old[r + n][: lst.d])
            elif r >= 1:
                assert torch.equal(x, y)


SIZES = [[40_000, 1, 333], [700_000, 63, 7]]


# blocks that a CTA holds, that a cluster holds, and blocks of the two-pass pipeline
@pytest.mark.parametrize("k", [10, 14, 16, 20])
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("feedback", [True, False])
@pytest.mark.parametrize("max_norm", [math.inf, 5.0])
@pytest.mark.parametrize("value", [math.nan, -math.inf])
def test_training_goes_on_as_if_the_round_had_not_been(k, sizes, feedback, max_norm, value):
    from paper_2302_08545_b200 import runner, thc

    def train(rounds, bad=None):
        ctx = context(k=k)
        grads = T.make(sizes, ["f32", "bf16"], 3, seed=1)
        weights = T.make(sizes, ["bf16"], 1, seed=2)
        tr, wl = runner.TensorRound(ctx, grads, error_feedback=feedback), thc.Tensors(ctx, weights)
        m, v, master = (torch.zeros(wl.d, device="cuda") for _ in range(3))
        lr, step = torch.full((1,), 0.1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
        seen = {}
        for rnd in rounds:
            fresh = T.make(sizes, ["f32", "bf16"], 3, seed=10 + rnd)
            if rnd == bad:
                fresh[1][0][12_345] = value
            for w, f in zip(grads, fresh):
                for x, y in zip(w, f):
                    x.copy_(y)
            every = [m, v, master, step, *weights[0], *(tr.ef or [])]
            held = [x.clone() for x in every]
            out = tr.run(rnd, max_norm=max_norm)
            tr.adamw(wl, lr, step, m, v, master=master, max_norm=1.0, weight_decay=0.1)
            status = ctx.status()
            if rnd == bad:
                assert bool(torch.isnan(out).all()) and status & thc.STATUS_NONFINITE
                assert all(torch.equal(x, y) for x, y in zip(every, held))
                back = thc.Tensors(ctx, T.make(sizes, ["bf16"], 1))
                tr.scatter(back, max_norm=max_norm)        # a program with an optimizer of its own sees it
                assert all(bool(torch.isnan(x).all()) for x in back.tensors[0]) and ctx.status() != 0
            else:
                assert bool(torch.isfinite(out).all()) and not status & thc.STATUS_NONFINITE
                assert not torch.equal(master, held[2])
            seen[rnd] = [out.clone()] + [x.clone() for x in every]
        return seen

    got, without = train((0, 1, 2, 3), bad=1), train((0, 2, 3))
    for rnd, every in without.items():
        assert all(torch.equal(x, y) for x, y in zip(got[rnd], every)), rnd


def test_bf16_rounds_and_a_captured_step():
    """The flag is looked at when a captured step is replayed, not when it is captured."""
    from paper_2302_08545_b200 import runner, thc
    ctx = context(n=2, k=10, in_dtype=1)
    sizes = [5000, 77]
    grads, weights = T.make(sizes, ["bf16"], 2, seed=1), T.make(sizes, ["f32"], 1, seed=2)
    tr, wl = runner.TensorRound(ctx, grads), thc.Tensors(ctx, weights)
    m, v = (torch.zeros(wl.d, device="cuda") for _ in range(2))
    lr, step = torch.full((1,), 0.1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")

    def call():
        tr.run(1, max_norm=1.0)
        tr.adamw(wl, lr, step, m, v, max_norm=0.5)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    held = [x.clone() for x in (m, v, *weights[0])]
    good = grads[1][1][5].clone()
    grads[1][1][5] = math.nan
    graph.replay()
    assert int(step) == 1 and ctx.status() & thc.STATUS_NONFINITE
    assert all(torch.equal(x, y) for x, y in zip((m, v, *weights[0]), held))
    grads[1][1][5] = good
    graph.replay()
    assert int(step) == 2 and not ctx.status() & thc.STATUS_NONFINITE


def test_step_tensors_of_one_rank():
    import os
    import socket

    import torch.distributed as dist
    from paper_2302_08545_b200 import thc
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
        grads = T.make([40_000, 333], ["bf16", "f32"], 1, seed=5)
        lst = thc.Tensors(ctx, grads)
        ops = CudaOps(ctx, lst.d, dev)
        dp = DataParallelRound(ops, lst.d, 12, 4, ctx.sizes(lst.d, 1).acc_bits)
        ef = torch.zeros(lst.d, device=dev)
        out = dp.step_tensors(lst, 0, max_norm=3.0, ef=ef)[0]
        assert bool(torch.isfinite(out).all()) and bool(ef.any()) and ctx.status() == 0
        held, good = ef.clone(), grads[0][1][7].clone()
        grads[0][1][7] = math.inf
        out = dp.step_tensors(lst, 1, max_norm=3.0, ef=ef)[0]
        assert bool(torch.isnan(out).all()) and torch.equal(ef, held) and ctx.status() & thc.STATUS_NONFINITE
        grads[0][1][7] = good
        again = dp.step_tensors(lst, 2, max_norm=3.0, ef=ef)[0].clone()
        ef.copy_(held)
        assert torch.equal(dp.step_tensors(lst, 2, max_norm=3.0, ef=ef)[0], again) and not ctx.status() & thc.STATUS_NONFINITE
    finally:
        dist.destroy_process_group()


@pytest.mark.parametrize("k", [10, 14, 16, 20])
def test_finite_gradients_past_what_the_transform_holds(k):
    """Not clipped, a norm above 2^126 / (sqrt(B) t_p) makes a round void and leaves the residuals finite; up to there, and clipped at any
    norm, the round is served: values of one kind, of random signs, and a single one."""
    from paper_2302_08545_b200 import runner, thc, workloads as W
    ctx = context(n=2, k=k)
    limit = 2.0 ** 126 / (2.0 ** (k / 2) * W.T_P["1/32"])
    size = 3 * (1 << min(k, 16))
    grads = T.make([size, 77], ["f32"], 2, seed=1)
    signs = torch.randn(size, device="cuda")
    kinds = [torch.ones(size, device="cuda"), signs, torch.nn.functional.one_hot(torch.tensor(5), size).float().cuda()]
    for kind in kinds:
        tr = runner.TensorRound(ctx, grads, error_feedback=True)
        unit = (kind.double() / torch.linalg.vector_norm(kind.double())).float()
        for x in (grads[0][1], grads[1][1]):
            x.zero_()
        rnd = 0
        for norm, max_norm, void in ((0.99 * limit, math.inf, False), (1.01 * limit, math.inf, True), (1.01 * limit, 1.0, False), (2e38, math.inf, True),
                                     (2e38, 1.0, False), (2e38, 2.0 * limit, True), (1.0, math.inf, False)):
            grads[0][0].copy_(unit * norm)
            grads[1][0].copy_(signs * 1e-3)
            held = [x.clone() for x in tr.ef]
            for e in tr.ef if not void else []:
                e.zero_()                          # (a residual of a step at the limit would be added to the next one)
            out = tr.run(rnd, max_norm=max_norm)
            flags = ctx.status()
            assert all(bool(torch.isfinite(e).all()) for e in tr.ef), (norm, max_norm)
            if void:
                assert bool(torch.isnan(out).all()) and flags & thc.STATUS_NONFINITE
                assert all(torch.equal(x, y) for x, y in zip(tr.ef, held))
            else:
                assert bool(torch.isfinite(out).all()) and not flags & thc.STATUS_NONFINITE
            rnd += 1
