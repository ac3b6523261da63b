"""Lists of tensors on the GPU: norm, clipping, the ways into and out of the flat vector and the Adam step against
their definitions in 64 bits.

Bounds, with u = 2^-24: fp32 squares are added in fp64.  Eight exact squares of 16-bit values are added in fp32 in three
levels, each of which is off by at most u of a sum of positive terms, 3 u in all, and then in fp64; the norm, a square root, is
off by half of that, before(list) = 1.5 u, or 0 without 16-bit tensors.  It is rounded to fp32 (u).  The factor is formed in fp64
from the norm before that rounding, so it is off by before(list), and rounded (u); the product is rounded (u), then once more to
the tensor's type.  The Adam step's bounds are beside its test."""
import gc
import math

import pytest
import torch

import tensor_lists as T
from tensor_lists import TYPES, U

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def nothing_left_behind():
    """What a caught exception's frames hold (tensors) goes with the test, not in the middle of a later one."""
    yield
    gc.collect()


EDGES = [1, 7, 0, 8, 9, 63, 64, 65, 255, 1000, 2047, 2048, 2049, 4096 + 17, 100_003]
SMALL = 1.0 + 2.0 ** -16               # second-order terms of the bounds


def context(in_dtype="f32", **kw):
    from paper_2302_08545_b200 import thc, workloads as W
    return thc.Context(**dict(dict(bits=4, granularity=30, table=W.TABLES[(4, 30)], t_p=2.0, log2_block=12, seed=1,
                                   in_dtype=thc.THC_BF16 if in_dtype == "bf16" else thc.THC_F32), **kw))


def setup(workers, in_dtype="f32"):
    from paper_2302_08545_b200 import thc
    ctx = context(in_dtype)
    lst = thc.Tensors(ctx, workers)
    norms = torch.full((lst.n,), -1.0, device="cuda")
    ws = torch.empty(lst.workspace_bytes, dtype=torch.uint8, device="cuda")
    return ctx, lst, norms, ws


def before(workers):
    return 0.0 if all(x.dtype == torch.float32 for x in workers[0]) else 1.5 * U


def check_norms(norms, workers):
    ref = torch.tensor([T.norm(w) for w in workers], dtype=torch.float64)
    T.within(norms.cpu(), ref, ref * (before(workers) + U) * SMALL)
    return ref.tolist()


LISTS = [
    ([1], ["f32"], 1, 0), ([1], ["f16"], 3, 1), ([5], ["bf16"], 1, 3), (EDGES, ["f32"], 1, 0), (EDGES, ["bf16"], 2, 0),
    (EDGES, ["f16"], 1, 0), (EDGES, ["f32", "bf16", "f16", "bf16"], 3, 0), (EDGES, ["f32"], 2, 1), (EDGES, ["bf16"], 1, 4),
    (EDGES, ["f16"], 2, 2), (EDGES, ["f16", "f32"], 1, 5), ([300_001, 2_000_003], ["f32"], 5, 0), ([7_000_003], ["bf16"], 1, 0),
    ([17] * 400, ["f32", "bf16"], 2, 0), ([4096] * 64, ["bf16"], 64, 0), ([2000, 100, 7], ["f32", "f16"], 64, 0), ([131_072], ["f32"], 1, 0),
    ([131_073], ["f32"], 1, 0), ([1025] * 64, ["bf16"], 3, 0), ([8_388_608], ["bf16"], 1, 0), ([8_388_609], ["f32"], 1, 0), ([20_000_001, 9], ["f16"], 1, 0),
]


@pytest.mark.parametrize("sizes,types,n,shift", LISTS)
def test_norm(sizes, types, n, shift):
    workers = T.make(sizes, types, n, shift, seed=len(sizes) + n)
    ctx, lst, norms, ws = setup(workers)
    ws.fill_(0xA5)
    ctx.grad_norm(lst, norms, ws)
    check_norms(norms, workers)
    first = norms.clone()
    ctx.grad_norm(lst, norms, ws)
    assert torch.equal(first, norms) and ctx.status() == 0


@pytest.mark.parametrize("sizes,types,n,shift", LISTS)
@pytest.mark.parametrize("in_place", [False, True])
def test_clip(sizes, types, n, shift, in_place):
    from paper_2302_08545_b200 import thc
    workers = T.make(sizes, types, n, shift, seed=3)
    old = [[x.clone() for x in w] for w in workers]
    ctx, lst, norms, ws = setup(workers)
    most = 0.7 * T.norm(workers[0])        # clips some workers or all
    outs = workers if in_place else T.make(sizes, types, n, shift + 1 if shift else 0, seed=9)
    ctx.clip_grads(lst, most, norms, ws, out=None if in_place else thc.Tensors(ctx, outs))
    ref = check_norms(norms, old)
    for w, o, r in zip(old, outs, ref):
        c = T.factor(r, most)
        for x, y in zip(w, o):
            exact = x.double() * c
            rel, least = T.half_step(y.dtype)
            T.within(y, exact, exact.abs() * ((before(old) + 2 * U + (rel if y.dtype != torch.float32 else 0)) * SMALL) + least + 2.0 ** -149)
    if not in_place:
        for w, b in zip(workers, old):
            assert all(torch.equal(x, y) for x, y in zip(w, b))


def test_clip_leaves_what_is_around_the_tensors_alone():
    room = torch.full((20_000,), 5.0, dtype=torch.bfloat16, device="cuda")
    pieces, at = [], 3
    for s in (1, 9, 2047, 4099, 64, 5):
        pieces.append(room[at: at + s])
        at += s + 2
    ctx, lst, norms, ws = setup([pieces])
    ctx.clip_grads(lst, 1.0, norms, ws)
    inside = torch.zeros_like(room, dtype=torch.bool)
    for p in pieces:
        inside[p.storage_offset(): p.storage_offset() + p.numel()] = True
    assert bool((room[~inside] == 5.0).all()) and bool((room[inside] < 5.0).all())


@pytest.mark.parametrize("below", [True, False])
def test_a_norm_below_the_bound_changes_nothing(below):
    workers = T.make(EDGES, ["f32", "bf16", "f16"], 2, seed=4)
    old = [[x.clone() for x in w] for w in workers]
    ctx, lst, norms, ws = setup(workers)
    ctx.clip_grads(lst, 1e9 if below else math.inf, norms, ws)
    assert all(torch.equal(x, y) for w, b in zip(workers, old) for x, y in zip(w, b))
    check_norms(norms, old)


def test_max_norm_zero_and_zero_gradients():
    workers = T.make([100, 3000], ["f32"], 1, seed=4)
    ctx, lst, norms, ws = setup(workers)
    ctx.clip_grads(lst, 0.0, norms, ws)
    assert all(not bool(x.any()) for x in workers[0])
    ctx.clip_grads(lst, 1.0, norms, ws)
    assert float(norms) == 0.0 and all(not bool(x.any()) for x in workers[0]) and ctx.status() == 0


# lists that take the cluster, sums that the products add themselves, sums that the last CTA adds
LENGTHS = [[100, 5000], [100, 700_000], [100, 5_000_000]]


@pytest.mark.parametrize("sizes", LENGTHS)
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite(value, sizes):
    from paper_2302_08545_b200 import thc
    workers = T.make(sizes, ["f32", "bf16"], 3, seed=4)
    workers[1][1][4321] = value
    old = [[x.clone() for x in w] for w in workers]
    ctx, lst, norms, ws = setup(workers)
    ctx.clip_grads(lst, 1.0, norms, ws)
    assert ctx.status() == thc.STATUS_NONFINITE and ctx.status() == 0
    got = norms.tolist()
    assert math.isfinite(got[0]) and math.isfinite(got[2]) and (math.isnan(got[1]) if math.isnan(value) else got[1] == math.inf)
    for x, y in zip(workers[1], old[1]):
        if math.isnan(value):
            assert bool(torch.isnan(x).all())
        else:
            assert torch.equal(torch.isnan(x), torch.isinf(y)) and not bool(x[~torch.isnan(x)].any())
    for i in (0, 2):
        assert all(bool(torch.isfinite(x).all()) for x in workers[i])


def test_values_whose_squares_leave_fp32():
    """3e38 and 1e-30: their squares are neither in fp32's range; fp64 holds them."""
    x = torch.full((5000,), 1e-30, device="cuda")
    ctx, lst, norms, ws = setup([[x]])
    ctx.clip_grads(lst, 1.0, norms, ws)
    check_norms(norms, [[torch.full((5000,), 1e-30)]])
    x.fill_(3e38)
    y = x.clone()
    ctx.clip_grads(lst, 2.0, norms, ws)
    assert math.isinf(float(norms)) and ctx.status() == 0      # past fp32, not past fp64
    exact = y.double() * (2.0 / (math.sqrt(5000) * float(y[0].double()) + 1e-6))
    T.within(x, exact, exact.abs() * 2 * U * SMALL)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_squares_of_16_bits_at_the_ends_of_their_range(dtype):
    """Units whose squares leave fp32's range, next to ordinary ones, zeros and denormals; and all of one kind."""
    values = [3e38, 1e30, 1e-30, 1e-38, 1e-40, 0.0, 1.0, -2e19, 5e-20] if dtype == "bf16" else [65504.0, 6e-8, 6.1e-5, 0.0, 1.0, -3e-6]
    rows = [[v] * 8 for v in values] + [[v] * 3 + [values[0]] + [0.0] * 4 for v in values] + [[0.0] * 7 + [v] for v in values]
    for chosen in [rows, rows[1:], rows[2:5] * 9, rows[3:6] * 9] + [[r] * 40 for r in rows]:
        x = torch.tensor(chosen, dtype=torch.float64, device="cuda").to(TYPES[dtype]).reshape(-1)
        for pieces in ([x], [x, torch.zeros(5000, dtype=x.dtype, device="cuda")]):
            ctx, lst, norms, ws = setup([pieces])
            ctx.grad_norm(lst, norms, ws)
            ref = T.norm(pieces)
            if ref > 3.4e38:
                assert math.isinf(float(norms))
            else:
                T.within(norms.cpu(), torch.tensor([ref], dtype=torch.float64), torch.tensor([ref * 2.5 * U * SMALL + 2.0 ** -150], dtype=torch.float64))
            assert ctx.status() == 0


@pytest.mark.parametrize("flat", ["f32", "bf16", "residual", "residual in place"])
@pytest.mark.parametrize("sizes,types,n,shift", LISTS)
def test_gather(sizes, types, n, shift, flat):
    workers = T.make(sizes, types, n, shift, seed=5)
    ctx, lst, norms, ws = setup(workers, "bf16" if flat == "bf16" else "f32")
    most = 0.7 * T.norm(workers[0])
    dt = torch.bfloat16 if flat == "bf16" else torch.float32
    room = torch.full((n, lst.d + 64), 7.0, device="cuda", dtype=dt)
    flats = [row[: lst.d] for row in room]
    ef, e64 = None, [torch.zeros(lst.d, dtype=torch.float64, device="cuda")] * n
    if flat.startswith("residual"):
        ef = flats if flat.endswith("place") else [torch.empty(lst.d, device="cuda") for _ in range(n)]
        for e in ef:
            e.normal_()
        e64 = [e.double() for e in ef]
    ctx.gather_grads(lst, most, flats, norms, ws, ef=ef)
    ref = check_norms(norms, workers)
    for w, y, e, r in zip(workers, flats, e64, ref):
        c = T.factor(r, most)
        exact, product = e.clone(), torch.zeros_like(e)
        for x, o, v in zip(w, lst.offsets, lst.views(product)):
            v.copy_(x.double() * c)
        exact += product
        rel = T.half_step(dt)[0]
        # factor: before(list) + u of the product; one rounding of the result (fp32: of the product or of the fused sum)
        bound = product.abs() * (before(workers) + U) + exact.abs() * (U + (rel if flat == "bf16" else 0))
        T.within(y, exact, bound * SMALL + 2.0 ** -149)
        T.within(y[product == 0], e[product == 0], torch.zeros_like(e[product == 0]))
    assert bool((room[:, lst.d:] == 7.0).all())


def test_gather_without_clipping_is_a_copy():
    workers = T.make(EDGES, ["f32", "f16"], 2, seed=5)
    ctx, lst, norms, ws = setup(workers)
    flats = [torch.full((lst.d,), 3.0, device="cuda") for _ in range(2)]
    ctx.gather_grads(lst, math.inf, flats, None, None)
    for w, f in zip(workers, flats):
        assert all(torch.equal(x.float(), v) for x, v in zip(w, lst.views(f)))
        inside = torch.zeros(lst.d, dtype=torch.bool, device="cuda")
        for v in lst.views(inside):
            v.fill_(True)
        assert not bool(f[~inside].any())
    workers[0][3][0] = math.nan            # no norm: other elements are not touched by it
    ctx.gather_grads(lst, math.inf, flats, None, None)
    assert int(torch.isnan(flats[0]).sum()) == 1 and ctx.status() == 0


@pytest.mark.parametrize("sizes,types,n,shift", [c for c in LISTS if c[2] < 5])
def test_scatter(sizes, types, n, shift):
    workers = T.make(sizes, types, 1, shift, seed=6)
    ctx, lst, norms, ws = setup(workers)
    flat = torch.randn(lst.d, device="cuda")
    old = flat.clone()
    views = lst.views(flat)
    most = 0.5 * T.norm(views)
    ctx.scatter_grads(flat, most, lst, norms, ws)
    r, = check_norms(norms, [views])       # what is between the tensors does not count
    for x, v in zip(workers[0], views):
        exact = v.double() * T.factor(r, most)
        rel, least = T.half_step(x.dtype)
        T.within(x, exact, exact.abs() * ((2 * U + (rel if x.dtype != torch.float32 else 0)) * SMALL) + least + 2.0 ** -149)
    assert torch.equal(flat, old)
    ctx.scatter_grads(flat, math.inf, lst, None, None)
    assert all(torch.equal(x, v.to(x.dtype)) for x, v in zip(workers[0], views))


def test_scatter_to_places_in_the_flat_vector_itself():
    from paper_2302_08545_b200 import thc
    sizes = [100, 5000, 63]
    ctx, lst, norms, ws = setup(T.make(sizes, ["f32"], 1))
    flat = torch.randn(lst.d, device="cuda")
    old = flat.clone()
    own = thc.Tensors(ctx, [lst.views(flat)])
    ctx.scatter_grads(flat, 1.0, own, norms, ws)
    r, = check_norms(norms, [lst.views(old)])
    exact = old.double()
    for v in lst.views(exact):
        v.mul_(T.factor(r, 1.0))
    T.within(flat, exact, exact.abs() * 2 * U * SMALL)


def adam_exact(g, m, v, w, c, t, lr, wd, b1, b2, eps):
    """The step in 64 bits and bounds for m, v, w.  With u per rounding and per rounded constant: g = c x is 2 u off;
    m = fma(b1, m, a1 g): u |b1 m| (b1) + 4 u |a1 g| (g, a1, product) + u |m|.  v is a sum of positive terms, the larger
    error of which is a2 g g with 2 x 2 u (g), u (a2), 2 u (products): at most 7 u v + u v.  The denominator's root has half of
    v's and its own (5 u), its factor u, eps u, the sum u: at most 8 u.  The quotient adds 1 u and m's own error, the step
    size 1 u; keep = 1 - lr wd and its product 2 u |w|, the result u."""
    g = g * c
    m2 = b1 * m + (1 - b1) * g
    v2 = b2 * v + (1 - b2) * g * g
    root = torch.sqrt(v2 / (1 - b2 ** t)) + eps
    size = lr / (1 - b1 ** t)
    w2 = w * (1 - lr * wd) - size * m2 / root
    dm = U * ((b1 * m).abs() + 4 * ((1 - b1) * g).abs() + m2.abs())
    dw = size / root * dm + 10 * U * (size * m2 / root).abs() + U * (2 * w.abs() + w2.abs())
    least = 2.0 ** -140                    # denormals
    return m2, v2, w2, dm * SMALL + least, 8 * U * v2 * SMALL + least, dw * SMALL + least


@pytest.mark.parametrize("master", [True, False])
@pytest.mark.parametrize("sizes,types,shift", [([1], ["f32"], 0), (EDGES, ["f32"], 0), (EDGES, ["f32"], 3), (EDGES, ["bf16"], 0),
                                               (EDGES, ["bf16", "f32", "f16"], 0), (EDGES, ["f16", "f32", "bf16"], 1),
                                               ([3_000_001, 77], ["bf16"], 0), ([17] * 300, ["bf16", "f32"], 0)])
@pytest.mark.parametrize("per_tensor", [True, False])
def test_adamw(sizes, types, shift, master, per_tensor):
    if not master and types != ["f32"]:
        pytest.skip("without master weights the tensors are fp32")
    workers = T.make(sizes, types, 1, shift, seed=7, scale=0.1)
    ctx, lst, norms, ws = setup(workers)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    flat = lambda: torch.randn(lst.d, device="cuda", generator=gen)  # noqa: E731
    grad, m, v = flat(), flat() * 0.1, flat().square() * 0.01
    wm = flat() if master else None
    lr, step = torch.full((1,), 1e-2, device="cuda"), torch.full((1,), 4, dtype=torch.int64, device="cuda")
    decay = torch.arange(len(sizes), device="cuda").float() * 0.01 if per_tensor else None
    b1, b2, eps = 0.9, 0.99, 1e-6
    inside = torch.zeros(lst.d, dtype=torch.bool, device="cuda")
    for x in lst.views(inside):
        x.fill_(True)
    for t in (5, 6, 7):
        old = [x.clone() for x in (m, v)] + ([wm.clone()] if master else [])
        weights = [x.double() for x in (lst.views(wm) if master else workers[0])]
        wide = [x.double() for x in (grad, m, v)]
        most = 0.5 * T.norm(lst.views(grad)) if t < 7 else math.inf
        ctx.adamw(grad, lst, lr, step, m, v, norms, ws, master=wm, decay=decay, betas=(b1, b2), eps=eps, weight_decay=0.05, max_norm=most)
        assert int(step) == t
        r, = check_norms(norms, [lst.views(grad)])
        for i, x in enumerate(workers[0]):
            g0, m0, v0 = (lst.views(y)[i] for y in wide)
            wd = float(decay[i]) if per_tensor else 0.05
            m2, v2, w2, dm, dv, dw = adam_exact(g0, m0, v0, weights[i], T.factor(r, most), t, float(lr), wd, b1, b2, eps)
            T.within(lst.views(m)[i], m2, dm)
            T.within(lst.views(v)[i], v2, dv)
            if master:
                T.within(lst.views(wm)[i], w2, dw)
                assert torch.equal(x, lst.views(wm)[i].to(x.dtype))
            else:
                T.within(x, w2, dw)
        for y, o in zip([m, v] + ([wm] if master else []), old):
            assert torch.equal(y[~inside], o[~inside])


@pytest.mark.parametrize("size", [5000, 700_000, 9_000_001])
def test_adamw_skips_a_step_whose_norm_is_not_finite(size):
    from paper_2302_08545_b200 import thc
    workers = T.make([size, 10], ["bf16"], 1)
    ctx, lst, norms, ws = setup(workers)
    grad = torch.randn(lst.d, device="cuda")
    grad[lst.offsets[1] - 1] = math.nan    # between the tensors: does not matter
    m, v, w = (torch.rand(lst.d, device="cuda") for _ in range(3))
    lr, step = torch.full((1,), 1e-2, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    ctx.adamw(grad, lst, lr, step, m, v, norms, ws, master=w, max_norm=1.0)
    assert int(step) == 1 and ctx.status() == 0
    held = [x.clone() for x in (m, v, w, *workers[0])]
    for bad in (math.nan, math.inf):
        grad[5] = bad
        ctx.adamw(grad, lst, lr, step, m, v, norms, ws, master=w, max_norm=1.0)
        assert int(step) == 1 and ctx.status() == thc.STATUS_NONFINITE
        assert all(torch.equal(x, y) for x, y in zip(held, (m, v, w, *workers[0])))


def test_other_addresses():
    """Gradients that are allocated anew: the list takes the new addresses from then on."""
    sizes, types = [100, 3000, 1] * 200, ["f32", "bf16"]   # more addresses than one launch takes
    first, second = T.make(sizes, types, 2, seed=1), T.make(sizes, types, 2, seed=2, shift=1)
    ctx, lst, norms, ws = setup(first)
    ctx.grad_norm(lst, norms, ws)
    check_norms(norms, first)
    lst.assign(second)
    ctx.grad_norm(lst, norms, ws)
    check_norms(norms, second)
    with pytest.raises(ValueError):
        lst.assign([first[0]])
    with pytest.raises(ValueError):
        lst.assign([[x.double() for x in w] for w in first])
    ctx.grad_norm(lst, norms, ws)
    check_norms(norms, second)


def test_captured_and_replayed_on_another_stream():
    workers = T.make([5000, 64, 100_001], ["bf16"], 1, seed=3)
    ctx, lst, norms, ws = setup(workers)
    grad = torch.randn(lst.d, device="cuda")
    state = [torch.rand(lst.d, device="cuda") for _ in range(3)]
    lr, step = torch.full((1,), 1e-2, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")

    def call():
        m, v, w = state
        ctx.adamw(grad, lst, lr, step, m, v, norms, ws, master=w, max_norm=1.0)
    held = [x.clone() for x in (*state, *workers[0])]
    for k in range(3):
        if k == 2:
            lr.fill_(5e-3)
        call()
    torch.cuda.synchronize()
    expected = [x.clone() for x in (*state, *workers[0])]
    for x, y in zip((*state, *workers[0]), held):
        x.copy_(y)
    step.zero_()
    lr.fill_(1e-2)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    for k in range(3):
        if k == 2:
            lr.fill_(5e-3)
        graph.replay()
    torch.cuda.synchronize()
    assert int(step) == 3
    assert all(torch.equal(x, y) for x, y in zip((*state, *workers[0]), expected))


def test_refused_arguments():
    from paper_2302_08545_b200 import thc
    workers = T.make([100, 300], ["f32"], 2)
    ctx, lst, norms, ws = setup(workers)
    one = thc.Tensors(ctx, workers[:1])
    half = thc.Tensors(ctx, T.make([100, 300], ["bf16"], 1))
    flat = lambda n=1: [torch.zeros(lst.d, device="cuda") for _ in range(n)]  # noqa: E731
    f = flat(2)
    lr, step = torch.ones(1, device="cuda"), torch.ones(1, dtype=torch.int64, device="cuda")
    g, m, v, w = flat(4)
    inf = math.inf

    def code(call):
        with pytest.raises(thc.ThcError) as e:
            call()
        return e.value.code
    EINVAL = thc.THC_EINVAL
    assert code(lambda: ctx.grad_norm(lst, norms, ws[:64])) == thc.THC_EWORKSPACE
    assert code(lambda: ctx.grad_norm(lst, None, ws)) == EINVAL
    assert code(lambda: ctx.grad_norm(lst, norms, None)) == EINVAL
    assert code(lambda: ctx.clip_grads(lst, -1.0, norms, ws)) == EINVAL
    assert code(lambda: ctx.clip_grads(lst, math.nan, norms, ws)) == EINVAL
    assert code(lambda: ctx.clip_grads(one, 1.0, norms, ws, out=half)) == EINVAL
    assert code(lambda: ctx.clip_grads(lst, 1.0, norms, ws, out=one)) == EINVAL
    assert code(lambda: ctx.clip_grads(lst, 1.0, None, ws)) == EINVAL
    # the same tensor twice, and an output that lies across an input
    twice = thc.Tensors(ctx, [[workers[0][0], workers[0][0]]])
    ctx.grad_norm(twice, norms, ws)
    assert code(lambda: ctx.clip_grads(twice, 1.0, norms, ws)) == EINVAL
    room = torch.zeros(1000, device="cuda")
    a, b = thc.Tensors(ctx, [[room[:100], room[200:500]]]), thc.Tensors(ctx, [[room[8:108], room[600:900]]])
    assert code(lambda: ctx.clip_grads(a, 1.0, norms, ws, out=b)) == EINVAL
    same = thc.Tensors(ctx, [[room[:100], room[600:900]]])
    ctx.clip_grads(a, 1.0, norms, ws, out=same)
    assert code(lambda: ctx.gather_grads(lst, 1.0, f, None, None)) == EINVAL
    assert code(lambda: ctx.gather_grads(lst, 1.0, [f[0], f[0]], norms, ws)) == EINVAL
    assert code(lambda: ctx.gather_grads(lst, 1.0, f, norms, ws, ef=[f[1], f[0]])) == EINVAL
    assert code(lambda: ctx.gather_grads(lst, 1.0, [f[0], None], norms, ws)) == EINVAL
    assert code(lambda: ctx.gather_grads(thc.Tensors(ctx, [[f[0][:100], f[1][:300]]]), 1.0, f[:1], norms, ws)) == EINVAL
    wide = context("bf16")
    assert code(lambda: wide.gather_grads(thc.Tensors(wide, workers), 1.0, [x.bfloat16() for x in f], norms, ws, ef=f)) == thc.THC_EUNSUPPORTED
    assert code(lambda: ctx.scatter_grads(f[0], 1.0, lst, norms, ws)) == EINVAL             # two workers
    assert code(lambda: ctx.scatter_grads(f[0], 1.0, thc.Tensors(ctx, [[f[0][4:104], f[0][128:428]]]), norms, ws)) == EINVAL
    step_ok = dict(betas=(0.9, 0.99), max_norm=inf)
    assert code(lambda: ctx.adamw(g, half, lr, step, m, v, norms, ws, **step_ok)) == EINVAL  # no master weights
    assert code(lambda: ctx.adamw(g, lst, lr, step, m, v, norms, ws, master=w, **step_ok)) == EINVAL
    assert code(lambda: ctx.adamw(g, one, lr, step, m, m, norms, ws, **step_ok)) == EINVAL
    assert code(lambda: ctx.adamw(g, one, lr, step, m, v, norms, ws, master=g, **step_ok)) == EINVAL
    assert code(lambda: ctx.adamw(g, one, None, step, m, v, norms, ws, **step_ok)) == EINVAL
    for bad in (dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(betas=(math.nan, 0.9)), dict(eps=-1.0), dict(eps=inf),
                dict(weight_decay=-1.0), dict(weight_decay=math.nan), dict(max_norm=math.nan)):
        assert code(lambda: ctx.adamw(g, one, lr, step, m, v, norms, ws, **dict(step_ok, **bad))) == EINVAL
    # what the library cannot see from an address
    for call in (lambda: ctx.grad_norm(lst, norms[:1], ws), lambda: ctx.grad_norm(lst, norms.double(), ws),
                 lambda: ctx.grad_norm(lst, norms.cpu(), ws),
                 lambda: ctx.gather_grads(lst, 1.0, [x[:-1] for x in f], norms, ws), lambda: ctx.gather_grads(lst, 1.0, f[:1], norms, ws),
                 lambda: ctx.gather_grads(lst, 1.0, [x.bfloat16() for x in f], norms, ws),
                 lambda: ctx.gather_grads(lst, 1.0, f, norms, ws, ef=[x[:-1] for x in f]),
                 lambda: ctx.scatter_grads(torch.zeros(2 * lst.d, device="cuda")[::2], 1.0, one, norms, ws),
                 lambda: ctx.adamw(g, one, lr, step.int(), m, v, norms, ws), lambda: ctx.adamw(g, one, lr, step, m[:-1], v, norms, ws),
                 lambda: ctx.adamw(g, one, lr, step, m, v, norms, ws, decay=lr),
                 lambda: thc.Tensors(ctx, [[room[::2]]]), lambda: thc.Tensors(ctx, [[room.double()]]), lambda: thc.Tensors(ctx, [[room.cpu()]]),
                 lambda: thc.Tensors(ctx, [[room], [room[:-1]]]), lambda: thc.Tensors(ctx, [[room], [room, room]]), lambda: thc.Tensors(ctx, []),
                 lambda: thc.Tensors(ctx, [[]])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(thc.ThcError):
        thc.Tensors(ctx, [[torch.zeros(0, device="cuda")]])
    half.close()
    with pytest.raises(ValueError):
        ctx.clip_grads(one, 1.0, norms, ws, out=half)
    assert code(lambda: ctx.grad_norm(half, norms, ws)) == EINVAL
    torch.cuda.synchronize()


@pytest.mark.parametrize("at", [4, 8])
@pytest.mark.parametrize("sizes", [[5000, 33], [300_001, 33]])
def test_vectors_that_start_at_16_bytes(sizes, at):
    """16 bytes are what the calls ask for; units of fp32 are 32."""
    from paper_2302_08545_b200 import thc
    workers = T.make(sizes, ["bf16", "f32"], 1, seed=3)
    ctx, lst, norms, ws = setup(workers)
    vectors = [torch.rand(lst.d + 8, device="cuda")[at: at + lst.d] for _ in range(6)]
    g, m, v, w, x, e = vectors
    e0 = e.double()
    ctx.gather_grads(lst, 10.0, [x], norms, ws, ef=[e])
    r, = check_norms(norms, workers)
    for t, y, z in zip(workers[0], lst.views(x), lst.views(e0)):
        product = t.double() * T.factor(r, 10.0)
        T.within(y, product + z, (product.abs() * 2.5 * U + (product + z).abs() * U) * SMALL + 2.0 ** -149)
    m0, v0, w0 = m.double(), v.double(), w.double()
    lr, step = torch.full((1,), 1e-2, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    ctx.adamw(g, lst, lr, step, m, v, norms, ws, master=w, betas=(0.9, 0.99), eps=1e-6, max_norm=1.0)
    r, = check_norms(norms, [lst.views(g)])
    for i, t in enumerate(workers[0]):
        m2, v2, w2, dm, dv, dw = adam_exact(*(lst.views(y)[i] for y in (g.double(), m0, v0, w0)), T.factor(r, 1.0), 1, float(lr), 0.0, 0.9, 0.99, 1e-6)
        T.within(lst.views(m)[i], m2, dm)
        T.within(lst.views(v)[i], v2, dv)
        T.within(lst.views(w)[i], w2, dw)
        assert torch.equal(t, lst.views(w)[i].to(t.dtype))
    ctx.scatter_grads(w, math.inf, lst, None, None)
    assert all(torch.equal(t, y.to(t.dtype)) for t, y in zip(workers[0], lst.views(w)))


def test_positions_past_32_bits():
    """More than 2^31 elements of 16 bits and 2^33 bytes of fp32 before the last tensors."""
    big = 2 ** 31 + 2049
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    x = torch.empty(big, dtype=torch.bfloat16, device="cuda")
    for part in x.split(1 << 28):
        part.normal_()
    workers = [[x, torch.randn(1000, device="cuda"), torch.randn(77, device="cuda").half()]]
    ctx, lst, norms, ws = setup(workers)
    flat = torch.full((lst.d,), 9.0, device="cuda")
    ctx.gather_grads(lst, 1000.0, [flat], norms, ws)
    square = sum(float((p.double() ** 2).sum()) for t in workers[0] for p in t.split(1 << 26))
    norm = math.sqrt(square)
    assert abs(float(norms) - norm) <= norm * 2.6 * U
    c = T.factor(norm, 1000.0)
    for t, v in zip(workers[0], lst.views(flat)):
        for a, b in zip(t.split(1 << 28), v.split(1 << 28)):
            exact = a.double() * c
            T.within(b, exact, exact.abs() * 4.6 * U + 2.0 ** -149)
    assert not bool(flat[big: lst.offsets[1]].any())
    back = [[torch.zeros_like(x), torch.zeros(1000, device="cuda"), torch.zeros(77, device="cuda").half()]]
    from paper_2302_08545_b200 import thc
    ctx.scatter_grads(flat, math.inf, thc.Tensors(ctx, back), None, None)
    for t, v in zip(back[0], lst.views(flat)):
        for a, b in zip(t.split(1 << 28), v.split(1 << 28)):
            assert torch.equal(a, b.to(a.dtype))


def test_values_past_the_end_of_16_bits():
    """fp32 values that fp16 and bf16 do not hold become infinite, as a rounding to nearest says."""
    from paper_2302_08545_b200 import thc
    workers = [[torch.zeros(100, device="cuda").half(), torch.zeros(100, device="cuda").bfloat16(), torch.zeros(100, device="cuda")]]
    ctx, lst, norms, ws = setup(workers)
    flat = torch.zeros(lst.d, device="cuda")
    for v in lst.views(flat):
        v[:4] = torch.tensor([65519.0, 65520.0, -7e4, 3.4e38], device="cuda")
    ctx.scatter_grads(flat, math.inf, lst, norms, ws)
    for x, v in zip(workers[0], lst.views(flat)):
        assert torch.equal(x, v.to(x.dtype))
    assert ctx.status() == 0


@pytest.mark.parametrize("steps", [0, 1, 1000, 10 ** 6, 2 ** 40])
@pytest.mark.parametrize("size", [100, 300_000])
def test_adamw_after_many_steps(steps, size):
    """1 - beta^t after few and very many steps."""
    workers = T.make([size], ["f32"], 1, seed=7)
    ctx, lst, norms, ws = setup(workers)
    grad, m, v = (torch.rand(lst.d, device="cuda") + 0.5 for _ in range(3))
    w0, m0, v0 = workers[0][0].double(), lst.views(m)[0].double(), lst.views(v)[0].double()
    lr, step = torch.full((1,), 1e-2, device="cuda"), torch.full((1,), steps, dtype=torch.int64, device="cuda")
    ctx.adamw(grad, lst, lr, step, m, v, norms, ws, betas=(0.9, 0.999), eps=1e-8, max_norm=math.inf)
    assert int(step) == steps + 1
    m2, v2, w2, dm, dv, dw = adam_exact(lst.views(grad)[0].double(), m0, v0, w0, 1.0, steps + 1, float(lr), 0.0, 0.9, 0.999, 1e-8)
    T.within(lst.views(m)[0], m2, dm)
    T.within(lst.views(v)[0], v2, dv)
    T.within(workers[0][0], w2, dw)


def test_many_calls_in_a_row_of_every_length():
    """Clusters, sums that the products add themselves and sums that the last CTA adds, one after the other on one context, with
    nothing between: every call's norm is its own."""
    from paper_2302_08545_b200 import thc
    ctx = context()
    cases = []
    for i, size in enumerate([100, 5_000_000, 70_000, 9_000_001, 131_073, 3]):
        workers = T.make([size, 65], ["f32", "bf16"], 1 + i % 3, seed=i)
        lst = thc.Tensors(ctx, workers)
        cases.append((workers, lst, [torch.empty(lst.d, device="cuda") for _ in workers]))
    ws = torch.empty(max(c[1].workspace_bytes for c in cases), dtype=torch.uint8, device="cuda")
    norms = torch.zeros(40, len(cases), 3, device="cuda")
    for r in range(40):
        for i, (workers, lst, flats) in enumerate(cases):
            ctx.gather_grads(lst, 1.0, flats, norms[r, i, : lst.n], ws)
    for i, (workers, lst, flats) in enumerate(cases):
        ref = torch.tensor([T.norm(w) for w in workers], dtype=torch.float64)
        T.within(norms[0, i, : lst.n].cpu(), ref, ref * 2.6 * U)
        assert bool((norms[:, i] == norms[0, i]).all())
    assert ctx.status() == 0


def test_two_contexts_on_two_streams():
    """The same list at the same time from two contexts, each with a stream and a workspace of its own; the stream given, or the
    current one."""
    from paper_2302_08545_b200 import thc
    for sizes in ([3000, 70], [2_000_003, 70], [9_000_001, 5]):
        workers = T.make(sizes, ["f32", "bf16"], 1, seed=6)
        first, second = context(), context()
        lst = thc.Tensors(first, workers)
        calls = []
        for ctx in (first, second):
            stream = torch.cuda.Stream()
            calls.append((ctx, stream, torch.empty(lst.workspace_bytes, dtype=torch.uint8, device="cuda"), torch.zeros(30, 1, device="cuda"),
                          torch.empty(lst.d, device="cuda")))
        torch.cuda.synchronize()
        for r in range(30):
            for i, (ctx, stream, ws, norms, flat) in enumerate(calls):
                if i == 0:
                    ctx.gather_grads(lst, 1.0 + i, [flat], norms[r], ws, stream=stream)
                else:
                    with torch.cuda.stream(stream):
                        ctx.gather_grads(lst, 1.0 + i, [flat], norms[r], ws)
        torch.cuda.synchronize()
        for i, (ctx, stream, ws, norms, flat) in enumerate(calls):
            r, = check_norms(norms[0], workers)
            assert bool((norms == norms[0]).all()) and ctx.status() == 0
            for x, y in zip(workers[0], lst.views(flat)):
                exact = x.double() * T.factor(r, 1.0 + i)
                T.within(y, exact, exact.abs() * (before(workers) + 2 * U) * SMALL + 2.0 ** -149)


def test_twenty_thousand_tensors():
    """More tensors than CTAs, most of them shorter than a unit or empty, pieces of one allocation in an order of their own."""
    from paper_2302_08545_b200 import thc
    n = 20_000
    sizes = [(7 * i) % 40 if i % 5 else 0 for i in range(n)]
    sizes[12_345] = 100_000
    ends = torch.tensor(sizes).cumsum(0).tolist()
    room = torch.randn(ends[-1], device="cuda")
    order = sorted(range(n), key=lambda i: (i * 7919) % n)
    pieces = [room[ends[i] - sizes[i]: ends[i]] for i in order]
    ctx, lst, norms, ws = setup([pieces])
    flat = torch.full((lst.d,), 5.0, device="cuda")
    ctx.gather_grads(lst, math.inf, [flat], norms, ws)
    check_norms(norms, [[room]])
    joined = torch.cat(pieces)
    places = torch.cat([torch.arange(o, o + p.numel()) for o, p in zip(lst.offsets, pieces)]).cuda()
    assert torch.equal(flat[places], joined)
    flat[places] = 0.0
    assert not bool(flat.any())
    moved = torch.randn_like(room)
    lst.assign([[moved[p.storage_offset(): p.storage_offset() + p.numel()] for p in pieces]])
    ctx.clip_grads(lst, 1.0, norms, ws)
    assert abs(float(torch.linalg.vector_norm(moved.double())) - 1.0) < 1e-5


def test_a_list_that_goes_during_a_capture():
    """Destroying one list does not spoil a capture of calls on another."""
    from paper_2302_08545_b200 import thc
    workers = T.make([5000, 64], ["f32"], 1, seed=3)
    ctx, lst, norms, ws = setup(workers)
    other = thc.Tensors(ctx, T.make([100], ["f32"], 1))
    ctx.grad_norm(lst, norms, ws)
    norms.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.grad_norm(lst, norms, ws)
        other.close()
        ctx.grad_norm(lst, norms, ws)
    graph.replay()
    torch.cuda.synchronize()
    check_norms(norms, workers)
