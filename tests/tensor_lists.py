"""Lists of tensors for the tests, and the definitions of the calls that take them, in 64 bits."""
import math

import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24                         # half a step of fp32


def half_step(dtype):
    """(relative, absolute): the most that one rounding to dtype is off."""
    info = torch.finfo(dtype)
    return info.eps / 2, info.smallest_normal * info.eps / 2


def make(sizes, types, n=1, shift=0, device="cuda", seed=0, scale=1.0):
    """n workers' tensors; each in an allocation of its own, `shift` + 0, 1, 2, ... elements from its start when
    shift is not 0."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    out = []
    for _ in range(n):
        pieces = []
        for i, s in enumerate(sizes):
            at = (shift + i) % 9 if shift else 0
            room = torch.zeros(s + at, dtype=TYPES[types[i % len(types)]], device=device)
            x = room[at:]
            x.copy_(torch.randn(s, generator=gen, device=device, dtype=torch.float64) * scale * (1 + i % 3))
            pieces.append(x)
        out.append(pieces)
    return out


def norm(pieces):
    return math.sqrt(math.fsum(float((x.double() ** 2).sum()) for x in pieces))


def factor(norm, max_norm):
    if math.isinf(max_norm):
        return 1.0
    return min(1.0, max_norm / (norm + 1e-6)) if norm == norm else norm


def within(got, ref, bound):
    """got (any type) against ref and bound (float64)."""
    d = (got.double() - ref).abs()
    assert bool((d <= bound).all()), f"off by {float((d / bound.clamp(min=1e-300)).max())} of the bound"
