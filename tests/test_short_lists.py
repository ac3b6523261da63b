"""The lists of test_gpu_short_lists.py take the cluster (on a fake CUDA runtime, as in test_launch_host.py)."""
import pytest
import torch

import short_lists as S
from test_launch_host import child  # noqa: F401  (a fixture)
from test_tensors import LISTS

if torch.cuda.is_available():
    pytest.skip("for machines without a device", allow_module_level=True)


def test_they_are_one_launch(child):  # noqa: F811
    assert S.pieces(S.SIXTEEN) == 16 and S.pieces(S.SIXTY_FOUR) == 64
    lists = [(sizes, n) for sizes, _, n, _ in S.LISTS]
    assert max(S.pieces(s) for s, _ in lists) == 64
    child(LISTS + f"""
lists, sixteen = {lists!r}, {S.SIXTEEN!r}
fl = p(*[(1 << 46) + (i << 34) for i in range(64)])
rows = lambda: [("cluster" in r[1], r[2], r[5]) for r in log() if r[0] == "launch" and "list_pieces" not in r[1]]
b = context(10, in_dtype=1)
for sizes, n in lists:
    h, one, out = lst(sizes, [0] * len(sizes), n), lst(sizes, [1] * len(sizes)), lst(sizes, [0] * len(sizes), n, at=1 << 43)
    hb = lst(sizes, [1] * len(sizes), n, ctx=b)
    log()
    assert call("thc_grad_norm", h, N) == 0 and call("thc_clip_grads", h, 1.0, None, N) == 0 and call("thc_clip_grads", h, 1.0, out, N) == 0
    assert call("thc_gather_grads", h, 1.0, None, fl, N) == 0 and call("thc_gather_grads", h, 1.0, fl, fl, N) == 0
    assert L.thc_gather_grads(b._h, hb, 1.0, None, fl, N, WS, 1 << 30, None) == 0
    assert call("thc_scatter_grads", 1 << 50, 1.0, one, N) == 0
    assert rows() == [(True, 8, 8)] * 7
    if sum(-(-s // 2048) for s in sizes) <= 16:
        conf = thc._AdamwConfig(0.9, 0.99, 1e-8, 0.1, 1.0)
        F = [(1 << 52) + (i << 40) for i in range(4)]
        assert L.thc_adamw(c._h, ctypes.byref(conf), F[0], one, 1 << 47, 1 << 48, F[3], F[1], F[2], None, N, WS, 1 << 30, None) == 0
        assert rows() == [(True, 8, 8)]
""")
