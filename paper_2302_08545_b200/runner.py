"""Buffer management around the C-ABI calls: allocate a round's device buffers with torch
and issue prepare / compress / aggregate / decompress in order.  No arithmetic here."""
from __future__ import annotations

import math

import numpy as np
import torch

from . import thc
from .workloads import Workload


def context_for(w: Workload, workers: int | None = None, acc_bits: int = 0,
                exact_range: bool = False) -> thc.Context:
    return thc.Context(bits=w.bits, granularity=w.granularity, table=w.table, t_p=w.t_p,
                       log2_block=w.log2_block, seed=w.seed,
                       in_dtype=thc.THC_BF16 if w.in_dtype == "bf16" else thc.THC_F32,
                       workers=w.n if workers is None else workers, acc_bits=acc_bits,
                       range_mode=1 if exact_range else 0)


class Round:
    """Device buffers of one simulated cluster: n gradient buffers in one GPU's memory."""

    def __init__(self, ctx: thc.Context, n: int, d: int, in_dtype: str = "f32",
                 device: str = "cuda:0", want_rotated: bool = False):
        self.ctx, self.n, self.d = ctx, n, d
        self.sz = ctx.sizes(d, n)
        dev = torch.device(device)
        self.device = dev
        gdt = torch.float32 if in_dtype == "f32" else torch.bfloat16
        self.grads = [torch.zeros(d, dtype=gdt, device=dev) for _ in range(n)]
        self.scales = torch.zeros(self.sz.scales_count, dtype=torch.float32, device=dev)
        self.packed = [torch.zeros(self.sz.packed_bytes, dtype=torch.uint8, device=dev)
                       for _ in range(n)]
        self.total = torch.zeros(self.sz.sum_bytes, dtype=torch.uint8, device=dev)
        self.out = torch.zeros(d, dtype=torch.float32, device=dev)
        self.workspace = torch.zeros(self.sz.workspace_bytes, dtype=torch.uint8, device=dev)
        self.rotated = ([torch.zeros(self.sz.d_pad, dtype=torch.float32, device=dev)
                         for _ in range(n)] if want_rotated else None)

    # -- host <-> device helpers (copies only)
    def upload(self, x: np.ndarray):
        """x: [n, d] float32, or uint16 bf16 bit patterns for bf16 contexts."""
        for i in range(self.n):
            t = torch.from_numpy(np.ascontiguousarray(x[i]))
            if self.grads[i].dtype == torch.bfloat16:
                t = t.view(torch.int16).view(torch.bfloat16) if t.dtype != torch.bfloat16 else t
            self.grads[i].copy_(t)

    def sum_numpy(self) -> np.ndarray:
        dt = {8: np.uint8, 16: np.uint16, 32: np.uint32}[self.sz.acc_bits]
        return self.total.cpu().numpy().view(dt)

    # -- the four calls
    def prepare(self, stream=None):
        self.ctx.prepare(self.grads, self.d, self.scales, self.workspace, stream)

    def prepare_minmax(self, rnd: int = 0, stream=None):
        self.ctx.prepare_minmax(self.grads, self.d, rnd, self.scales, self.workspace,
                                rotated=self.rotated, stream=stream)

    def compress(self, rnd: int = 0, stream=None):
        self.ctx.compress(self.grads, self.d, rnd, self.scales, self.packed, self.workspace,
                          rotated=self.rotated, stream=stream)

    def prepare_compress(self, rnd: int = 0, stream=None):
        self.ctx.prepare_compress(self.grads, self.d, rnd, self.scales, self.packed, self.workspace,
                                  rotated=self.rotated, stream=stream)

    def quantize_rotated(self, rnd: int = 0, stream=None):
        self.ctx.quantize_rotated(self.rotated, self.d, rnd, self.scales, self.packed, stream=stream)

    def aggregate(self, stream=None):
        self.ctx.aggregate(self.packed, self.d, self.total, stream)

    def decompress(self, rnd: int = 0, stream=None):
        self.ctx.decompress(self.total, self.n, self.d, rnd, self.scales, self.out,
                            self.workspace, stream)

    def aggregate_decompress(self, rnd: int = 0, want_sums: bool = False, stream=None):
        self.ctx.aggregate_decompress(self.packed, self.d, rnd, self.scales, self.out, self.workspace,
                                      total=self.total if want_sums else None, stream=stream)

    def run(self, rnd: int = 0, with_prepare: bool = True, stream=None, fused: bool = False):
        if with_prepare and fused:
            self.prepare_compress(rnd, stream)
        else:
            if with_prepare:
                self.prepare(stream)
            self.compress(rnd, stream)
        if fused:
            self.aggregate_decompress(rnd, want_sums=True, stream=stream)
        else:
            self.aggregate(stream)
            self.decompress(rnd, stream)


class TensorRound:
    """A round between a program's tensors, n workers' lists of them on one GPU: the gradients, clipped by each
    worker's norm, become the flat vectors that the round compresses; its average goes, clipped again, back to
    tensors (scatter) or through an Adam step into the weights (adamw).

    ``grads`` is a sequence of n sequences of tensors (see thc.Tensors), which the object keeps and reads every round: gradients
    that are allocated anew every step (torch's zero_grad sets them to None) are given to it by assign.  With error feedback each worker's
    residual of one round is added to its gradients of the next (fp32 contexts).

    A round in which a worker's norm is not finite (see thc_void_round for how large it may be) is void: its average is NaN in every element, so that adamw takes no step and
    scatter hands the NaN on, and every worker keeps its residual; the next round is as if it had not been."""

    def __init__(self, ctx: thc.Context, grads, error_feedback: bool = False):
        self.ctx = ctx
        self.grads = thc.Tensors(ctx, grads)
        n, d, device = self.grads.n, self.grads.d, grads[0][0].device
        self.round = Round(ctx, n, d, "bf16" if ctx.in_dtype == thc.THC_BF16 else "f32", device=device)
        self.norms = torch.zeros(n, dtype=torch.float32, device=device)
        self.average_norm = torch.zeros(1, dtype=torch.float32, device=device)
        self.workspace = torch.empty(self.grads.workspace_bytes, dtype=torch.uint8, device=device)    # serves every list
        self.ef = [torch.zeros(d, dtype=torch.float32, device=device) for _ in range(n)] if error_feedback else None

    def assign(self, grads, stream=None):
        """Other gradient tensors of the same shapes and types, for the rounds issued on ``stream`` from here on."""
        self.grads.assign(grads, stream)

    def _check(self, tensors: thc.Tensors):
        if tensors.n != 1 or not tensors.same_layout(self.grads):
            raise ValueError("a list of one worker with the places of the gradients in the flat vector is expected")

    def run(self, rnd: int = 0, max_norm: float = math.inf, stream=None):
        """Gather and the round; returns the flat average (a buffer of this object)."""
        r = self.round
        self.ctx.gather_grads(self.grads, max_norm, r.grads, self.norms, self.workspace, ef=self.ef, stream=stream)
        r.run(rnd, fused=True, stream=stream)
        self.ctx.void_round(self.grads, max_norm, self.norms, r.scales, r.out, None if self.ef is None else r.grads, self.ef, stream)
        if self.ef is not None:
            self.ctx.error_feedback(r.grads, r.packed, r.d, rnd, r.scales, self.ef, r.workspace, stream)
        return r.out

    def scatter(self, tensors: thc.Tensors, max_norm: float = math.inf, stream=None):
        """The average, clipped by its norm, to the tensors of a list with one worker and the gradients' sizes."""
        self._check(tensors)
        self.ctx.scatter_grads(self.round.out, max_norm, tensors, self.average_norm, self.workspace, stream)

    def adamw(self, weights: thc.Tensors, lr, step, m, v, master=None, stream=None, **how):
        """An Adam step with the average (arguments as thc.Context.adamw)."""
        self._check(weights)
        self.ctx.adamw(self.round.out, weights, lr, step, m, v, self.average_norm, self.workspace,
                       master=master, stream=stream, **how)
