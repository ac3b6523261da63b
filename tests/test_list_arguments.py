"""Workspaces of the calls on lists: the binding refuses what the library cannot see from an address."""
import pytest
import torch

from paper_2302_08545_b200 import thc
from test_tensors import context


def calls(c, t, ws):
    f, norms = [torch.zeros(t.d) for _ in range(4)], torch.zeros(1)
    lr, step = torch.zeros(1), torch.zeros(1, dtype=torch.int64)
    return (lambda: c.grad_norm(t, norms, ws, stream=0), lambda: c.clip_grads(t, 1.0, norms, ws, stream=0),
            lambda: c.gather_grads(t, 1.0, f[:1], norms, ws, stream=0), lambda: c.scatter_grads(f[0], 1.0, t, norms, ws, stream=0),
            lambda: c.adamw(f[0], t, lr, step, f[1], f[2], norms, ws, master=f[3], stream=0))


@pytest.mark.parametrize("table", [True, False])
def test_workspaces_that_the_binding_refuses(table, monkeypatch):
    """Not contiguous, expanded, or on another device; whether torch's table describes a tensor or its attributes are asked for."""
    c = context()
    t = thc.Tensors(c, [[torch.zeros(100)]])
    size = t.workspace_bytes

    class Plain(torch.Tensor):                  # (what the table does not describe)
        pass
    make = (lambda x: x) if table else (lambda x: x.as_subclass(Plain))
    elsewhere = torch.empty(size, dtype=torch.uint8, device="meta")
    for ws in (torch.zeros(2 * size, dtype=torch.uint8)[::2], torch.zeros(1, dtype=torch.uint8).expand(size),
               torch.zeros(size // 8 + 8, 8).t(), elsewhere):
        for call in calls(c, t, make(ws)):
            with pytest.raises((ValueError, BufferError, RuntimeError)) as e:
                call()
            assert not isinstance(e.value, thc.ThcError)
    for ws in (torch.zeros(size, dtype=torch.uint8), torch.zeros(size // 4, 1), torch.zeros(size // 8, dtype=torch.int64)):
        for call in calls(c, t, make(ws)):
            with pytest.raises(thc.ThcError) as e:      # served as far as a context without device goes
                call()
            assert e.value.code == thc.THC_ECUDA
