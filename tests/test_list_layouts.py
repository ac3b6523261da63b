"""Objects that lead from a round's average to tensors refuse lists that lie otherwise in the flat vector than the gradients."""
import pytest
import torch

from test_tensors import context


def test_lists_that_lie_otherwise_are_refused():
    from paper_2302_08545_b200 import runner, thc
    from paper_2302_08545_b200.data_parallel import CudaOps
    ctx = context()
    make = lambda *sizes: thc.Tensors(ctx, [[torch.zeros(s) for s in sizes]])  # noqa: E731
    tr = runner.TensorRound.__new__(runner.TensorRound)                # (no device to make its buffers on)
    tr.grads, tr.ctx = thc.Tensors(ctx, [[torch.zeros(100), torch.zeros(70)]] * 2), ctx
    ops = CudaOps(ctx, 256, torch.device("cpu"))
    ops._workspace_of(make(100, 70))
    workspace = ops._workspace_of(make(65, 128))                       # other sizes, the same places
    assert ops._workspace_of(make(100, 70)) is workspace
    lr, step = torch.zeros(1), torch.zeros(1, dtype=torch.int64)
    f = [torch.zeros(256) for _ in range(4)]
    for bad in (make(100, 64), make(70, 180), make(100, 70, 1), make(256), thc.Tensors(ctx, [[torch.zeros(100), torch.zeros(70)]] * 2)):
        for call in (lambda: tr.scatter(bad), lambda: tr.adamw(bad, lr, step, f[0], f[1], master=f[2]), lambda: ops.gather(bad),
                     lambda: ops.scatter(f[0], bad), lambda: ops.adamw(f[0], bad, lr, step, f[1], f[2])):
            with pytest.raises(ValueError):
                call()
