"""An assignment of addresses whose launches fail, on a fake CUDA runtime: the host's addresses and the device's table never
disagree in a call that is served."""
import os
import subprocess
import sys

import pytest
import torch

from test_launch_host import PRELUDE, ROOT
from test_tensors import LISTS

if torch.cuda.is_available():
    pytest.skip("for machines without a device", allow_module_level=True)

# A launch fails when `fake_fail_after` more have gone out.
FAILING = r"""
#define _GNU_SOURCE
#include <dlfcn.h>
int fake_fail_after = -1;
int cudaLaunchKernelExC(const void *c, const void *f, void **args)
{
    static int (*next)(const void *, const void *, void **);
    if (next == 0) next = (int (*)(const void *, const void *, void **))dlsym(RTLD_NEXT, "cudaLaunchKernelExC");
    if (fake_fail_after == 0) return 719;
    if (fake_fail_after > 0) --fake_fail_after;
    return next(c, f, args);
}
"""

CODE = LISTS + """
fail = ctypes.c_int.in_dll(fake, "fake_fail_after")
E = thc.THC_EINVAL
numel, k = [100] * 1000, 1000
h = lst(numel, [0] * k, at=1 << 33, step=1 << 12)
new = p(*[(1 << 40) + (i << 12) for i in range(k)])
def assign(after):
    fail.value = after
    rc = L.thc_tensors_assign(c._h, h, new, None)
    fail.value = -1
    return rc
old_place, new_place = (1 << 33) + 999 * 4096, (1 << 40) + 999 * 4096       # of the last tensor
gather = lambda flat: call("thc_gather_grads", h, 1.0, None, p(flat), N)
assert gather(old_place) == E and gather(new_place) == 0
# nothing was set: the list is as before
assert assign(0) == thc.THC_ECUDA
assert gather(old_place) == E and gather(new_place) == 0
# part of the table was set: no call is served before an assignment succeeds
assert assign(1) == thc.THC_ECUDA
clipped = lst(numel, [0] * k, at=1 << 41, step=1 << 12)
calls = [lambda: gather(1 << 50), lambda: call("thc_grad_norm", h, N), lambda: call("thc_clip_grads", h, 1.0, None, N),
         lambda: call("thc_clip_grads", clipped, 1.0, h, N), lambda: call("thc_scatter_grads", 1 << 50, 1.0, h, N),
         lambda: L.thc_void_round(c._h, h, 1.0, N, 1 << 51, 1 << 50, None, None, None)]
log()
assert [f() for f in calls] == [E] * len(calls) and log() == []
assert assign(0) == thc.THC_ECUDA and gather(1 << 50) == E
assert assign(-1) == 0 and gather(old_place) == 0 and gather(new_place) == E
assert [f() for f in calls] == [0] * len(calls)
"""


def test_launches_that_fail(tmp_path):
    fakes = []
    for name, source in (("failing", FAILING), ("fake_cudart", open(os.path.join(ROOT, "tests", "fake_cudart.c")).read())):
        c, so = tmp_path / f"{name}.c", tmp_path / f"{name}.so"
        c.write_text(source)
        subprocess.run([os.environ.get("CC", "gcc"), "-O1", "-fPIC", "-shared", "-I/usr/local/cuda/include", "-o", str(so), str(c), "-ldl"], check=True)
        fakes.append(str(so))
    res = subprocess.run([sys.executable, "-c", PRELUDE.format(root=ROOT) + CODE], capture_output=True, text=True,
                         env=dict(os.environ, LD_PRELOAD=":".join(fakes)), timeout=300)
    assert res.returncode == 0, res.stderr[-3000:]
