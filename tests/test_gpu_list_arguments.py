"""Workspaces of the calls on lists that are elsewhere or not contiguous are refused, other types of the right size are served."""
import pytest
import torch

import tensor_lists as T

pytestmark = pytest.mark.gpu


def test_workspaces():
    from paper_2302_08545_b200 import thc, workloads as W
    ctx = thc.Context(bits=4, granularity=30, table=W.TABLES[(4, 30)], t_p=2.0, log2_block=12, seed=1)
    workers = T.make([300_001, 7], ["f32"], 1)
    lst, norms = thc.Tensors(ctx, workers), torch.zeros(1, device="cuda")
    size = lst.workspace_bytes
    room = torch.zeros(2 * size, dtype=torch.uint8, device="cuda")
    for bad in (torch.zeros(size, dtype=torch.uint8), torch.zeros(size, dtype=torch.uint8).pin_memory(), room[::2], room[:1].expand(size)):
        with pytest.raises(ValueError):
            ctx.grad_norm(lst, norms, bad)
    with pytest.raises(thc.ThcError) as e:
        ctx.grad_norm(lst, norms, room[: size - 16])
    assert e.value.code == thc.THC_EWORKSPACE
    for good in (room[:size], room.view(torch.int64), torch.zeros(size // 4, 1, device="cuda")):
        norms.zero_()
        ctx.grad_norm(lst, norms, good)
        assert abs(float(norms) / T.norm(workers[0]) - 1.0) < 2.0 ** -23
    assert ctx.status() == 0
