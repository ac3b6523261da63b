"""The workspace of a round of tensors stays where a captured call wrote it."""
import pytest
import torch

import tensor_lists as T

pytestmark = pytest.mark.gpu


def test_a_captured_round_keeps_its_workspace():
    """Six workers of 60M elements (whose sums take fewer CTAs a worker than a list of one), the round captured alone, the Adam step
    called outside the graph."""
    from paper_2302_08545_b200 import runner, thc, workloads as W
    ctx = thc.Context(bits=4, granularity=30, table=W.TABLES[(4, 30)], t_p=W.T_P["1/32"], log2_block=12, seed=W.THC_SEED, workers=6)
    sizes = [60_000_000, 100]
    grads = T.make(sizes, ["bf16"], 6, seed=1)
    tr = runner.TensorRound(ctx, grads)
    weights = thc.Tensors(ctx, T.make(sizes, ["bf16"], 1, seed=2))
    master, m, v = (torch.zeros(weights.d, device="cuda") for _ in range(3))
    lr, step = torch.full((1,), 0.1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    tr.run(3, max_norm=1.0)
    expected, norms, address = tr.round.out.clone(), tr.norms.clone(), tr.workspace.data_ptr()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tr.run(3, max_norm=1.0)
    for k in range(2):
        tr.round.out.zero_()
        graph.replay()
        tr.adamw(weights, lr, step, m, v, master=master, max_norm=1.0)
        assert tr.workspace.data_ptr() == address
        assert torch.equal(tr.round.out, expected) and torch.equal(tr.norms, norms) and int(step) == k + 1
    assert ctx.status() == 0
