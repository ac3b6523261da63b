"""One workspace serves every list of a device (on a fake CUDA runtime, as in test_launch_host.py)."""
import pytest
import torch

from test_launch_host import child  # noqa: F401  (a fixture)
from test_tensors import LISTS

if torch.cuda.is_available():
    pytest.skip("for machines without a device", allow_module_level=True)


def test_the_workspace_of_one_worker_is_the_workspace_of_all(child):  # noqa: F811
    """For every number of workers and lengths on both sides of every limit of the launches: the same size, and the sums that the
    launched CTAs leave fit behind the results."""
    child(LISTS + """
rows = lambda: [r for r in log() if r[0] == "launch" and "list_norm" in r[1]]
fl = p(*[(1 << 55) + (i << 40) for i in range(64)])
limits = [1, 8, 16, 64, 592, 148 * 8, 4096, 592 * 8, 592 * 8 * 6, 592 * 8 * 48, 29_297, 70_000, 400_000]
sizes = thc._TensorsSizes()
seen = set()
for n in range(1, 65):
    for pieces in sorted({max(1, v // k + e) for v in limits for k in (1, n) for e in (-1, 0, 1)}):
        h = lst([2048 * pieces], [0], n, at=1 << 33, step=1 << 34)
        assert L.thc_tensors_sizes(h, ctypes.byref(sizes)) == 0
        seen.add(sizes.workspace_bytes)
        log()
        if pieces <= 80_000:
            assert L.thc_grad_norm(c._h, h, N, WS, sizes.workspace_bytes, None) == 0
            assert L.thc_gather_grads(c._h, h, 1.0, None, fl, N, WS, sizes.workspace_bytes, None) == 0
            for r in rows():
                assert 2048 + r[2] * n * 8 <= sizes.workspace_bytes, (n, pieces, r)
        L.thc_tensors_destroy(h)
assert len(seen) == 1, seen
""")
