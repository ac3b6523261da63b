"""The one-launch form of the calls on lists (a cluster per worker) with tensors at any address, of any type and of several workers: the
tests of test_gpu_tensors.py, whose odd lists are one piece too long for it.  test_short_lists.py checks that these lists take it."""
import gc

import pytest

import short_lists as S
import test_gpu_tensors as G

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def nothing_left_behind():
    yield
    gc.collect()


@pytest.mark.parametrize("sizes,types,n,shift", S.LISTS)
def test_norm(sizes, types, n, shift):
    G.test_norm(sizes, types, n, shift)


@pytest.mark.parametrize("sizes,types,n,shift", S.LISTS)
@pytest.mark.parametrize("in_place", [False, True])
def test_clip(sizes, types, n, shift, in_place):
    G.test_clip(sizes, types, n, shift, in_place)


@pytest.mark.parametrize("sizes,types,n,shift", S.LISTS)
@pytest.mark.parametrize("flat", ["f32", "bf16", "residual", "residual in place"])
def test_gather(sizes, types, n, shift, flat):
    G.test_gather(sizes, types, n, shift, flat)


@pytest.mark.parametrize("sizes,types,n,shift", S.LISTS)
def test_scatter(sizes, types, n, shift):
    G.test_scatter(sizes, types, n, shift)


@pytest.mark.parametrize("sizes", [S.SIXTEEN, [2049, 33], [5]])
@pytest.mark.parametrize("types,shift", [(["f32"], 0), (["f32"], 1), (["f32"], 3), (["f32"], 8), (["bf16"], 0), (["bf16"], 4), (["f16"], 1),
                                         (["f16", "f32", "bf16"], 5), (["bf16", "f32"], 2)])
@pytest.mark.parametrize("per_tensor", [True, False])
def test_adamw(sizes, types, shift, per_tensor):
    G.test_adamw(sizes, types, shift, True, per_tensor)
    if types == ["f32"]:
        G.test_adamw(sizes, types, shift, False, per_tensor)
