"""Finite gradients whose norm fp32 does not hold: the norm reads infinity, no status bit is set, and the calls clip by the fp64
norm; only a round that would send them is void."""
import math

import pytest
import torch

import tensor_lists as T
from test_gpu_tensors import SMALL, adam_exact, context, setup

pytestmark = pytest.mark.gpu


# lists that take the cluster, sums that the products add themselves, sums that the last CTA adds
@pytest.mark.parametrize("sizes", [[5000, 7], [700_001, 7], [9_000_001, 7]])
def test_the_adam_step_is_taken(sizes):
    workers = T.make(sizes, ["f32"], 1, seed=7)
    ctx, lst, norms, ws = setup(workers)
    grad = (torch.rand(lst.d, device="cuda") + 0.5) * 1.5e38
    m, v = torch.zeros(lst.d, device="cuda"), torch.zeros(lst.d, device="cuda")
    w0 = [x.double() for x in workers[0]]
    lr, step = torch.full((1,), 1e-2, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    norm = T.norm(lst.views(grad))
    assert 3.5e38 < norm < 1e43
    ctx.adamw(grad, lst, lr, step, m, v, norms, ws, betas=(0.9, 0.99), eps=1e-8, max_norm=100.0)
    assert math.isinf(float(norms)) and ctx.status() == 0 and int(step) == 1
    for i, x in enumerate(workers[0]):
        zero = torch.zeros(sizes[i], dtype=torch.float64, device="cuda")
        m2, v2, w2, dm, dv, dw = adam_exact(lst.views(grad)[i].double(), zero, zero, w0[i], T.factor(norm, 100.0), 1, float(lr), 0.0, 0.9, 0.99, 1e-8)
        T.within(lst.views(m)[i], m2, dm)
        T.within(lst.views(v)[i], v2, dv)
        T.within(x, w2, dw)


@pytest.mark.parametrize("sizes", [[5000, 7], [700_001, 7], [9_000_001, 7]])
def test_scatter_and_gather_clip_by_it(sizes):
    workers = T.make(sizes, ["f32"], 1, seed=7)
    ctx, lst, norms, ws = setup(workers)
    flat = (2.0 * torch.rand(lst.d, device="cuda") - 1.0) * 3e38
    norm = T.norm(lst.views(flat))
    ctx.scatter_grads(flat, 100.0, lst, norms, ws)
    assert math.isinf(float(norms)) and norm > 3.5e38 and ctx.status() == 0
    for x, v in zip(workers[0], lst.views(flat)):
        exact = v.double() * T.factor(norm, 100.0)
        T.within(x, exact, exact.abs() * 2 * T.U * SMALL + 2.0 ** -149)
    for x, v in zip(workers[0], lst.views(flat)):
        x.copy_(v)
    out = torch.zeros_like(flat)
    ctx.gather_grads(lst, 100.0, [out], norms, ws)
    assert math.isinf(float(norms)) and ctx.status() == 0
    for x, v in zip(lst.views(out), lst.views(flat)):
        exact = v.double() * T.factor(norm, 100.0)
        T.within(x, exact, exact.abs() * 2 * T.U * SMALL + 2.0 ** -149)


def test_a_round_that_would_send_them_is_void():
    from paper_2302_08545_b200 import runner, thc
    ctx = context()
    tr = runner.TensorRound(ctx, [[torch.full((5000,), 3e38, device="cuda")]], error_feedback=True)
    for max_norm in (math.inf, 1.0):
        assert bool(torch.isnan(tr.run(0, max_norm=max_norm)).all()) and math.isinf(float(tr.norms))
        assert not bool(tr.ef[0].any()) and ctx.status() & thc.STATUS_NONFINITE
