"""Lists of tensors without a GPU: layout, refusals (of the library, on a context without device, and of the binding), what
the calls launch (on a fake CUDA runtime, as in test_launch_host.py), and a round of several ranks that begins with tensors."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2302_08545_b200 import thc, workloads as W
from test_data_parallel import ROOT, WORKER, _free_port
from test_launch_host import child  # noqa: F401  (a fixture)

if torch.cuda.is_available():
    pytest.skip("for contexts without a device", allow_module_level=True)


def context(**kw):
    return thc.Context(**dict(dict(bits=4, granularity=30, table=W.TABLES[(4, 30)], t_p=2.0, log2_block=10, seed=1), **kw))


def create(ctx, addresses, numel, dtypes, n=1, count=None):
    """thc_tensors_create's return code and the list's handle."""
    count = len(numel) if count is None else count
    h = ctypes.c_void_p()
    rc = thc.lib().thc_tensors_create(ctx._h, (ctypes.c_void_p * len(addresses))(*addresses), (ctypes.c_uint64 * len(numel))(*numel),
                                      (ctypes.c_uint32 * len(dtypes))(*dtypes), n, count, ctypes.byref(h))
    return rc, h


def test_layout():
    c = context()
    shapes = [(3, 5), (64,), (0,), (65,), (2, 2048), (1,)]
    t = thc.Tensors(c, [[torch.zeros(s, dtype=d) for s, d in zip(shapes, [torch.float32, torch.bfloat16, torch.float16] * 2)] for _ in range(3)])
    assert t.offsets == [0, 64, 128, 128, 256, 4352] and t.d == 4416 and t.elements == 15 + 64 + 65 + 4096 + 1
    assert t.n == 3 and t.count == 6 and t.device == -1 and t.workspace_bytes > 0
    flat = torch.arange(t.d, dtype=torch.float32)
    views = t.views(flat)
    assert [tuple(v.shape) for v in views] == shapes
    assert float(views[3][0]) == 128.0 and float(views[4][1, 0]) == 256 + 2048 and float(views[5][0]) == 4352
    assert not any(o % thc.TENSOR_ALIGN for o in t.offsets) and t.d % thc.TENSOR_ALIGN == 0


def test_lists_that_are_refused():
    c = context()
    ok = [1 << 20]
    for args in [([0], [5], [0]), ([(1 << 20) + 2], [5], [0]), ([(1 << 20) + 1], [5], [1]), (ok, [5], [3]), (ok, [0], [0]),
                 (ok, [(1 << 40) + 1], [0])]:
        assert create(c, *args)[0] == thc.THC_EINVAL, args
    for kw in [dict(n=0), dict(n=65), dict(count=0), dict(count=(1 << 20) + 1)]:
        assert create(c, ok * 70, [5], [0], **kw)[0] == thc.THC_EINVAL
    assert create(c, ok * 64, [1 << 40], [0], n=64)[0] == thc.THC_EUNSUPPORTED
    rc, h = create(c, [0, (1 << 20) + 2], [0, 5], [0, 1])      # an empty tensor needs no address
    assert rc == thc.THC_OK and thc.lib().thc_tensors_destroy(h) == thc.THC_OK
    L = thc.lib()
    assert L.thc_tensors_create(c._h, None, None, None, 1, 1, ctypes.byref(h)) == thc.THC_EINVAL
    assert L.thc_tensors_sizes(None, None) == thc.THC_EINVAL and L.thc_tensors_offsets(None, None) == thc.THC_EINVAL
    assert L.thc_tensors_destroy(None) == thc.THC_OK


def test_calls_without_a_device_fail_loudly():
    c = context()
    t = thc.Tensors(c, [[torch.zeros(100)]])
    f, one, ws = [torch.zeros(t.d) for _ in range(4)], torch.zeros(1), torch.zeros(t.workspace_bytes, dtype=torch.uint8)
    for call in (lambda: c.grad_norm(t, one, ws, stream=0), lambda: c.clip_grads(t, 1.0, one, ws, stream=0),
                 lambda: c.gather_grads(t, 1.0, f[:1], one, ws, stream=0), lambda: c.scatter_grads(f[0], 1.0, t, one, ws, stream=0),
                 lambda: c.adamw(f[0], t, one, torch.zeros(1, dtype=torch.int64), f[1], f[2], one, ws, master=f[3], stream=0),
                 lambda: t.assign([[torch.zeros(100)]], stream=0)):
        with pytest.raises(thc.ThcError) as e:
            call()
        assert e.value.code == thc.THC_ECUDA


def test_tensors_that_the_binding_refuses():
    c = context()
    t = thc.Tensors(c, [[torch.zeros(100)], [torch.zeros(100)]])
    ws, norms = torch.zeros(t.workspace_bytes, dtype=torch.uint8), torch.zeros(2)
    f = [torch.zeros(t.d) for _ in range(2)]
    for call in (lambda: c.grad_norm(t, norms[:1], ws, stream=0), lambda: c.grad_norm(t, norms.double(), ws, stream=0),
                 lambda: c.grad_norm(t, torch.zeros(4)[::2], ws, stream=0),
                 lambda: c.gather_grads(t, 1.0, f[:1], norms, ws, stream=0), lambda: c.gather_grads(t, 1.0, f + f, norms, ws, stream=0),
                 lambda: c.gather_grads(t, 1.0, [x[:-1] for x in f], norms, ws, stream=0),
                 lambda: c.gather_grads(t, 1.0, [x.bfloat16() for x in f], norms, ws, stream=0),
                 lambda: c.gather_grads(t, 1.0, f, norms, ws, ef=f[:1], stream=0),
                 lambda: thc.Tensors(c, [[torch.zeros(9)[::2]]]), lambda: thc.Tensors(c, [[torch.zeros(9).double()]]),
                 lambda: thc.Tensors(c, [[torch.zeros(9)], [torch.zeros(8)]]), lambda: thc.Tensors(c, [[torch.zeros(9)], []]),
                 lambda: thc.Tensors(c, []), lambda: thc.Tensors(c, [[]]),
                 lambda: thc.Tensors(c, [[torch.zeros(9)], [torch.zeros(9).half()]])):
        with pytest.raises(ValueError):
            call()
    closed = thc.Tensors(c, [[torch.zeros(100)], [torch.zeros(100)]])
    closed.close()
    closed.close()
    with pytest.raises(ValueError):
        c.clip_grads(t, 1.0, norms, ws, out=closed, stream=0)
    with pytest.raises(thc.ThcError):
        c.grad_norm(closed, norms, ws, stream=0)
    with pytest.raises(TypeError):
        c._call.grad_norm(c._handle, t._handle)


LISTS = """
import math
c = context(10)
L = thc.lib()
def lst(numel, dtypes, n=1, at=1 << 33, step=1 << 30, ctx=c):
    h, k = ctypes.c_void_p(), len(numel)
    a = (ctypes.c_void_p * (n * k))(*[at + i * step for i in range(n * k)])
    rc = L.thc_tensors_create(ctx._h, a, (ctypes.c_uint64 * k)(*numel), (ctypes.c_uint32 * k)(*dtypes), n, k, ctypes.byref(h))
    assert rc == 0, rc
    return h
def p(*v): return (ctypes.c_void_p * len(v))(*v)
WS, N = 1 << 44, 1 << 45                # workspace, norms
def call(name, *args): return getattr(L, name)(c._h, *args, WS, 1 << 30, None)
"""


def test_which_kernels_the_calls_launch(child):  # noqa: F811
    """Short lists: one launch, a cluster of eight per worker.  Longer ones: sums, then products of eight pieces to a CTA.
    Without a norm the products alone."""
    child(LISTS + """
def rows():                             # but for the kernel that makes a list's table
    return [(r[1].split("kernel")[0].split("list_")[-1], r[2:]) for r in log() if r[0] == "launch" and "list_pieces" not in r[1]]
fl = p(*[(1 << 46) + (i << 34) for i in range(4)])
for n in (1, 4):
    h = lst([64 * 2048], [0], n)
    assert call("thc_gather_grads", h, 1.0, None, fl, N) == 0
    assert rows() == [("cluster_", [8, 512, 65536, 8])]
    assert call("thc_grad_norm", h, N) == 0
    assert rows() == [("cluster_", [8, 512, 0, 8])]
    h = lst([64 * 2048, 1], [0, 0], n)
    assert call("thc_gather_grads", h, 1.0, None, fl, N) == 0
    got = rows()
    assert [g[0] for g in got] == ["norm_", "product_"] and got[1][1][0] >= 65 * n // 8 and got[0][1][1] == got[1][1][1] == 256, got
    assert call("thc_gather_grads", h, math.inf, None, fl, None) == 0
    assert [g[0] for g in rows()] == ["product_"]
h = lst([300_000_001], [1])
assert call("thc_clip_grads", h, 1.0, None, N) == 0
got = rows()
assert got[0][1][:2] == [5 * 592, 256] and got[1][1][:2] == [-(-(-(-300_000_001 // 2048)) // 8), 256], got
assert call("thc_grad_norm", h, N) == 0
assert [(g[0], g[1][0]) for g in rows()] == [("norm_", 592)]
# addresses anew: 448 to a launch
h = lst([5] * 1000, [0] * 1000)
assert L.thc_tensors_assign(c._h, h, p(*[(1 << 40) + 64 * i for i in range(1000)]), None) == 0
assert [g[0] for g in rows()] == ["assign_"] * 3
""")


def test_refused_calls_launch_nothing(child):  # noqa: F811
    child(LISTS + """
E, U, S = thc.THC_EINVAL, thc.THC_EUNSUPPORTED, thc.THC_EWORKSPACE
nan, inf = math.nan, math.inf
h, h2 = lst([100, 70], [0, 0]), lst([100, 70], [0, 0], 2, at=1 << 40)
half = lst([100, 70], [1, 1], at=1 << 41)
F = [(1 << 46) + (i << 20) for i in range(8)]
assert call("thc_grad_norm", h, None) == E and call("thc_grad_norm", None, N) == E and call("thc_grad_norm", h, N + 2) == E
assert L.thc_grad_norm(None, h, N, WS, 1 << 30, None) == E
assert L.thc_grad_norm(c._h, h, N, None, 1 << 30, None) == E and L.thc_grad_norm(c._h, h, N, WS + 8, 1 << 30, None) == E
assert L.thc_grad_norm(c._h, h, N, WS, 8, None) == S
for bad in (-1.0, nan, -inf):
    assert call("thc_clip_grads", h, bad, None, N) == E and call("thc_gather_grads", h, bad, None, p(F[0]), N) == E
    assert call("thc_scatter_grads", F[0], bad, h, N) == E
assert call("thc_clip_grads", h, inf, None, None) == E
assert call("thc_clip_grads", h, 1.0, h2, N) == E and call("thc_clip_grads", h, 1.0, half, N) == E
# outputs over inputs: the same tensor is served, another place in it is not, nor one tensor twice
assert call("thc_clip_grads", h, 1.0, lst([100, 70], [0, 0]), N) == 0
assert call("thc_clip_grads", h, 1.0, lst([100, 70], [0, 0], at=(1 << 33) + 4), N) == E
assert call("thc_clip_grads", h, 1.0, lst([100, 70], [0, 0], at=(1 << 33) + (1 << 30), step=-(1 << 30)), N) == E
twice = lst([100, 70], [0, 0], step=0)
assert call("thc_grad_norm", twice, N) == 0 and call("thc_clip_grads", twice, 1.0, None, N) == E
g3 = lst([100, 70, 9], [0, 0, 0], at=1 << 42)
def create(places):
    h, k = ctypes.c_void_p(), 3
    rc = L.thc_tensors_create(c._h, p(*[(1 << 42) + v for v in places]), (ctypes.c_uint64 * k)(100, 70, 9), (ctypes.c_uint32 * k)(0, 0, 0), 1, k, ctypes.byref(h))
    assert rc == 0
    return h
G = 1 << 30
assert call("thc_clip_grads", g3, 1.0, create((0, 5 * G, 2 * G)), N) == 0          # two of them in place
assert call("thc_clip_grads", g3, 1.0, create((5 * G, 6 * G, 7 * G)), N) == 0      # none
assert call("thc_clip_grads", g3, 1.0, create((0, G, 2 * G + 4)), N) == E          # the last one beside its place
assert call("thc_clip_grads", g3, 1.0, create((0, 2 * G, 5 * G)), N) == E          # one over another
assert call("thc_clip_grads", g3, 1.0, create((5 * G, G - 4, 6 * G)), N) == E
assert call("thc_clip_grads", g3, 1.0, create((400, G, 2 * G)), N) == 0            # right behind the tensor
log()
assert call("thc_gather_grads", h, 1.0, None, p(F[0]), None) == E          # a bound needs the norm
assert call("thc_gather_grads", h, 1.0, None, None, N) == E and call("thc_gather_grads", h, 1.0, None, p(None), N) == E
assert call("thc_gather_grads", h, 1.0, None, p(F[0] + 4), N) == E
assert call("thc_gather_grads", h2, 1.0, None, p(F[0], F[0]), N) == E and call("thc_gather_grads", h2, 1.0, None, p(F[0], F[0] + 256), N) == E
assert call("thc_gather_grads", h, 1.0, None, p((1 << 33) - 128), N) == E  # over a tensor
assert call("thc_gather_grads", h2, 1.0, p(F[1], F[0]), p(F[0], F[1]), N) == E
assert call("thc_gather_grads", h, 1.0, p(F[0] + 16), p(F[0]), N) == E and call("thc_gather_grads", h, 1.0, p(None), p(F[0]), N) == E
b = context(10, in_dtype=1)
hb = lst([100], [1], ctx=b)
assert L.thc_gather_grads(b._h, hb, 1.0, p(F[1]), p(F[0]), N, WS, 1 << 30, None) == U
assert call("thc_scatter_grads", None, 1.0, h, N) == E and call("thc_scatter_grads", F[0], 1.0, h2, N) == E
assert call("thc_scatter_grads", F[0], 1.0, twice, N) == E and call("thc_scatter_grads", F[0], 1.0, h, None) == E
assert call("thc_scatter_grads", (1 << 33) - 256, 1.0, h, N) == E
def adam(cfg=(0.9, 0.99, 1e-8, 0.1, 1.0), g=F[0], t=h, lr=1 << 47, step=1 << 48, w=None, m=F[1], v=F[2], decay=None, norms=N, none=False):
    conf = thc._AdamwConfig(*cfg)
    return L.thc_adamw(c._h, None if none else ctypes.byref(conf), g, t, lr, step, w, m, v, decay, norms, WS, 1 << 30, None)
for bad in ((1.0, 0.9, 0, 0, 1), (-0.1, 0.9, 0, 0, 1), (0.9, 1.0, 0, 0, 1), (nan, 0.9, 0, 0, 1), (0.9, 0.9, -1, 0, 1), (0.9, 0.9, inf, 0, 1),
            (0.9, 0.9, nan, 0, 1), (0.9, 0.9, 0, -1, 1), (0.9, 0.9, 0, inf, 1), (0.9, 0.9, 0, 0, -1), (0.9, 0.9, 0, 0, nan)):
    assert adam(cfg=bad) == E, (bad, adam(cfg=bad))
assert adam(none=True) == E and adam(g=None) == E and adam(m=None) == E and adam(v=None) == E and adam(lr=None) == E and adam(step=None) == E
assert adam(norms=None) == E and adam(step=(1 << 48) + 4) == E and adam(lr=(1 << 47) + 2) == E and adam(decay=(1 << 47) + 2) == E
assert adam(t=half) == E and adam(t=h2, w=F[3]) == E and adam(t=twice, w=F[3]) == E
assert adam(m=F[0]) == E and adam(v=F[1]) == E and adam(v=F[1] + 512) == E and adam(w=F[0]) == E and adam(m=F[1] + 8) == E and adam(m=(1 << 33) - 256) == E
assert [r for r in log() if r[0] == "launch" and "list_pieces" not in r[1]] == []
assert adam() == 0 and adam(t=half, w=F[3]) == 0 and adam(cfg=(0.0, 0.0, 0.0, 0.0, inf)) == 0
# addresses that are refused leave the list as it was
assert L.thc_tensors_assign(c._h, h, p(1 << 40, 3), None) == E and L.thc_tensors_assign(c._h, h, None, None) == E
assert call("thc_clip_grads", h, 1.0, lst([100, 70], [0, 0]), N) == 0
""")


GATHER = r"""
class TensorOps(OracleOps):                        # the tensors are concatenated; no clipping
    def gather(self, tensors, max_norm, ef):
        self.asked = max_norm
        flat = torch.cat([t.reshape(-1) for t in tensors])
        return flat if ef is None else flat + ef
    def residual(self, grad, packed, rnd, scales, ef):
        z = O.unpack(np.array(packed.numpy()), (d + 255) // 256 * 256, 4)
        ef.copy_(torch.from_numpy(O.error_feedback(grad.numpy(), z, scales.numpy(), cfg, rnd)))

ops = TensorOps()
dp = DataParallelRound(ops, d, k, 4, w)
mine = torch.from_numpy(x[rank].copy())
ef = torch.zeros(d)
errors = np.zeros_like(x)
for rnd in (5, 6):
    out, scales, packed, total = dp.step_tensors([mine[:300].view(3, 100), mine[300:]], rnd, max_norm=2.5, ef=ef)
    xr = x + errors
    ref = O.thc_round(xr, cfg, rnd)
    assert ops.asked == 2.5 and np.array_equal(out.numpy().view(np.uint32), ref["out"].view(np.uint32))
    errors = np.stack([O.error_feedback(xr[i], O.unpack(ref["packed"][i], (d + 255) // 256 * 256, 4), ref["scales"], cfg, rnd)
                       for i in range(world)])
    assert np.array_equal(ef.numpy(), errors[rank])
out2, _, _, _ = dp.step_tensors([mine], 7)
assert ops.asked == float("inf") and np.array_equal(out2.numpy().view(np.uint32), O.thc_round(x, cfg, 7)["out"].view(np.uint32))
"""


@pytest.mark.parametrize("world", [2, 3])
def test_a_round_that_begins_with_tensors(tmp_path, world):
    head, tail = WORKER.split('if os.environ["THC_MODE"]')[0], "\ndist.barrier()" + WORKER.split("\ndist.barrier()")[1]
    script = tmp_path / "worker.py"
    script.write_text(head + GATHER + tail)
    env = dict(os.environ, THC_ROOT=ROOT, THC_OUT=str(tmp_path), THC_BLOCKS="7", MASTER_ADDR="127.0.0.1", OMP_NUM_THREADS="1")
    res = subprocess.run([sys.executable, "-m", "torch.distributed.run", "--nnodes=1", f"--nproc-per-node={world}", "--master-addr",
                          "127.0.0.1", "--master-port", str(_free_port()), str(script)], capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-3000:]
    assert all((tmp_path / f"rank{r}.ok").exists() for r in range(world))


def test_what_a_rank_refuses():
    from paper_2302_08545_b200.data_parallel import CudaOps
    c = context()
    ops = CudaOps(c, 128, torch.device("cpu"))
    for lists in ([[torch.zeros(129)]], [[torch.zeros(128)], [torch.zeros(128)]]):
        with pytest.raises(ValueError):
            ops.gather(thc.Tensors(c, lists))
