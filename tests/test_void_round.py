"""Rounds with a gradient that is not finite, without a GPU: across gloo ranks (per-rank steps bound to the oracle) and what
thc_void_round refuses (on a fake CUDA runtime, as in test_launch_host.py)."""
import os
import subprocess
import sys

import pytest
import torch

from test_data_parallel import ROOT, WORKER, _free_port
from test_launch_host import child  # noqa: F401  (a fixture)
from test_tensors import LISTS

if torch.cuda.is_available():
    pytest.skip("for machines without a device", allow_module_level=True)

VOID = r"""
class TensorOps(OracleOps):                        # tensors are concatenated, clipped by their norm
    def __init__(self):
        self.norm = torch.zeros(1)
    def gather(self, tensors, max_norm, ef):
        flat = torch.cat([t.reshape(-1) for t in tensors])
        norm = flat.double().square().sum().sqrt()
        self.norm[0] = norm.float()
        if max_norm != float("inf"):
            flat = (flat.double() * torch.clamp(max_norm / (norm + 1e-6), max=1.0)).float()
        return flat if ef is None else flat + ef
    def residual(self, grad, packed, rnd, scales, ef):
        z = O.unpack(np.array(packed.numpy()), (d + 255) // 256 * 256, 4)
        ef.copy_(torch.from_numpy(O.error_feedback(grad.numpy(), z, scales.numpy(), cfg, rnd)))
    def void(self, tensors, max_norm, norms, grad, scales, out, ef=None):      # the definition of thc_void_round
        if not bool(torch.isfinite(norms).all()):
            out.fill_(float("nan"))
            scales.zero_()
            if ef is not None:
                grad.copy_(ef)

def rounds(dp, numbers, feedback, max_norm, bad=None, value=None):
    ef, held, seen = torch.zeros(d) if feedback else None, None, {}
    for rnd in numbers:
        mine = torch.from_numpy((x[rank] * (1.0 + 0.1 * rnd)).astype(np.float32))
        if rnd == bad and rank == world - 1:
            mine[417] = value
        before = None if ef is None else ef.clone()
        out = dp.step_tensors([mine[:300], mine[300:]], rnd, max_norm=max_norm, ef=ef)[0].clone()
        if rnd == bad:
            assert bool(torch.isnan(out).all()), (rank, out)
            assert ef is None or torch.equal(ef, before)
        else:
            assert bool(torch.isfinite(out).all())
        seen[rnd] = (out, None if ef is None else ef.clone())
    return seen

def make():
    if os.environ["THC_MODE"] == "peer":
        return PeerMemoryRound(TensorOps(), FilePeers(), d, k, 4, w)
    return DataParallelRound(TensorOps(), d, k, 4, w)
dp, peer_count = make(), 0
for feedback in (True, False):
    for max_norm in (float("inf"), 3.0):
        without = rounds(dp, (0, 2, 3), feedback, max_norm)
        for value in (float("nan"), float("inf"), -float("inf")):
            got = rounds(dp, (0, 1, 2, 3), feedback, max_norm, 1, value)
            for rnd, (out, ef) in without.items():
                assert torch.equal(got[rnd][0], out), (rnd, value)
                assert ef is None or torch.equal(got[rnd][1], ef)
"""


@pytest.mark.parametrize("world,mode", [(2, "collective"), (3, "collective"), (2, "peer"), (3, "peer")])
def test_a_round_with_a_gradient_that_is_not_finite_is_void_on_every_rank(tmp_path, world, mode):
    head, tail = WORKER.split('if os.environ["THC_MODE"]')[0], "\ndist.barrier()" + WORKER.split("\ndist.barrier()")[1]
    script = tmp_path / "worker.py"
    script.write_text(head + VOID + tail)
    env = dict(os.environ, THC_ROOT=ROOT, THC_OUT=str(tmp_path), THC_BLOCKS="7", THC_MODE=mode, MASTER_ADDR="127.0.0.1", OMP_NUM_THREADS="1")
    res = subprocess.run([sys.executable, "-m", "torch.distributed.run", "--nnodes=1", f"--nproc-per-node={world}", "--master-addr",
                          "127.0.0.1", "--master-port", str(_free_port()), str(script)], capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-3000:]
    assert all((tmp_path / f"rank{r}.ok").exists() for r in range(world))


def test_refused_calls_launch_nothing(child):  # noqa: F811
    child(LISTS + """
E, U = thc.THC_EINVAL, thc.THC_EUNSUPPORTED
h, h2 = lst([100, 70], [0, 0]), lst([100, 70], [1, 0], 2, at=1 << 40)
F = [(1 << 46) + (i << 20) for i in range(8)]
S = 1 << 47                             # one scale: 256 elements in blocks of 2^10
def void(t=h, norms=N, scales=S, out=F[0], grads=None, ef=None, ctx=c, most=math.inf):
    return L.thc_void_round(ctx._h if ctx else None, t, most, norms, scales, out, grads, ef, None)
log()
assert void(ctx=None) == E and void(t=None) == E and void(most=-1.0) == E and void(most=math.nan) == E
assert void(norms=None) == E and void(norms=N + 2) == E and void(scales=None) == E and void(scales=S + 4) == E
assert void(out=None) == E and void(out=F[0] + 8) == E
assert void(grads=p(F[1])) == E and void(ef=p(F[1])) == E                  # one without the other
assert void(grads=p(None), ef=p(F[1])) == E and void(grads=p(F[1]), ef=p(F[2] + 4)) == E
for grads, ef in ((p(F[0]), p(F[1])), (p(F[1]), p(F[1])), (p(F[1]), p(F[0])), (p(F[1]), p(F[1] + 16)), (p(F[1]), p(S)), (p(N), p(F[2]))):
    assert void(grads=grads, ef=ef) == E
assert void(t=h2, grads=p(F[1], F[1]), ef=p(F[2], F[3])) == E and void(t=h2, grads=p(F[1], F[2]), ef=p(F[3], F[1])) == E
assert void(out=S) == E and void(out=N) == E and void(scales=N) == E
b = context(10, in_dtype=1)
hb = lst([100], [1], ctx=b)
assert [r for r in log() if r[0] == "launch" and "list_pieces" not in r[1]] == []
assert void(ctx=b, t=hb, grads=p(F[1]), ef=p(F[2])) == U and void(ctx=b, t=hb) == 0
assert void() == 0 and void(grads=p(F[1]), ef=p(F[2])) == 0
assert void(t=h2, grads=p(F[1], F[2]), ef=p(F[3], F[3])) == 0             # residuals are only read
rows = [r for r in log() if r[0] == "launch"]
assert len(rows) == 4 and all("void_round" in r[1] and r[2:4] == [1, 256] for r in rows), rows
big = lst([1 << 30], [0], at=1 << 50)
assert void(t=big, out=1 << 52, scales=1 << 53) == 0
assert [r[2:4] for r in log() if r[0] == "launch" and "void_round" in r[1]] == [[296, 256]]
""")


def test_tensors_that_the_binding_refuses():
    from paper_2302_08545_b200 import thc, workloads as W
    c = thc.Context(bits=4, granularity=30, table=W.TABLES[(4, 30)], t_p=2.0, log2_block=6, seed=1)
    t = thc.Tensors(c, [[torch.zeros(100)], [torch.zeros(100)]])
    f, norms, scales = [torch.zeros(t.d) for _ in range(5)], torch.zeros(2), torch.zeros(2)
    for call in (lambda: c.void_round(t, 1.0, norms[:1], scales, f[0], stream=0), lambda: c.void_round(t, 1.0, norms, scales[:1], f[0], stream=0),
                 lambda: c.void_round(t, 1.0, norms, scales, f[0][:-1], stream=0), lambda: c.void_round(t, 1.0, norms, scales, f[0].half(), stream=0),
                 lambda: c.void_round(t, 1.0, norms, scales, f[0], grads=f[1:2], ef=f[3:5], stream=0),
                 lambda: c.void_round(t, 1.0, norms, scales, f[0], grads=f[1:3], ef=[f[3], f[4][1:]], stream=0)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(thc.ThcError) as e:
        c.void_round(t, 1.0, norms, scales, f[0], grads=f[1:3], ef=f[3:5], stream=0)
    assert e.value.code == thc.THC_ECUDA
