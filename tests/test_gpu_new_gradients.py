"""A training loop whose gradients are allocated anew every step, as after zero_grad(set_to_none=True)."""
import pytest
import torch

import tensor_lists as T

pytestmark = pytest.mark.gpu


def test_rounds_of_gradients_that_autograd_allocates():
    """Each round is the round of the gradients of its own step: against an object made for them."""
    from paper_2302_08545_b200 import runner, thc, workloads as W
    ctx = thc.Context(bits=4, granularity=30, table=W.TABLES[(4, 30)], t_p=W.T_P["1/32"], log2_block=10, seed=W.THC_SEED, workers=2)
    sizes = [5000, 77, 300]
    workers = [[x.requires_grad_() for x in w] for w in T.make(sizes, ["f32", "bf16"], 2, seed=1)]

    def backward(rnd):
        for i, w in enumerate(workers):
            for x in w:
                x.grad = None                          # (what zero_grad does; the memory goes back to the allocator)
            sum(((1 + i + rnd) * x.float().square()).sum() for x in w).backward()
        return [[x.grad for x in w] for w in workers]
    tr, held, outs = None, [], []
    for rnd in range(3):
        grads = backward(rnd)
        if tr is None:
            tr = runner.TensorRound(ctx, grads)
        else:
            assert any(x.data_ptr() != y.data_ptr() for v, w in zip(grads, tr.grads.tensors) for x, y in zip(v, w))
            tr.assign(grads)
        outs.append(tr.run(rnd, max_norm=2.0).clone())
        ref = runner.TensorRound(ctx, [[x.clone() for x in w] for w in grads])
        assert torch.equal(ref.run(rnd, max_norm=2.0), outs[-1]) and torch.equal(ref.norms, tr.norms)
        norms = torch.tensor([T.norm([x.detach() for x in w]) for w in grads], dtype=torch.float64)
        T.within(tr.norms.cpu(), norms, norms * 2.6 * T.U)
        held.append(float(tr.norms[0]))
    assert held[0] < held[1] < held[2] and ctx.status() == 0
    with pytest.raises(ValueError):
        tr.assign([[x.detach()[:-1] for x in w] for w in workers])
