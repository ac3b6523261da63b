"""What stands around a round of gradient compression, as cases that can be timed and compared: a
program's many gradient tensors before it and its many weight tensors behind it.

  norm      the global L2 norm of each worker's tensors
  clip      the same, and every tensor times min(1, max_norm / (norm + 1e-6)), into tensors of the
            same types
  gather    the tensors, clipped, to the flat vector that the compression reads (with the residual of
            error feedback added where it is kept)
  scatter   the flat average that the decompression wrote, clipped, to tensors
  adamw     the flat average, clipped, through an Adam step with decoupled weight decay, with flat
            fp32 moments, and fp32 master weights unless the tensors are fp32 themselves

In a flat vector each tensor starts at a multiple of 64 elements.  A program's tensors of one type are
pieces of one allocation here, as in a bucket; `odd` ones start anywhere in it.
"""
import math

import numpy as np
import torch

own = False

ALIGN = 64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BETA1, BETA2, EPS, DECAY = 0.9, 0.95, 1e-8, 0.1


def _case(kind, n, d, count, dtype, max_norm=1.0, **more):
    return dict(dict(odd=False, flat="f32", feedback=False), kind=kind, n=n, d=d, count=count, dtype=dtype, max_norm=max_norm, **more)


def listed():
    return [
        # a few small layers: bound by latency
        _case("norm", 1, 3_000, 4, "f32", name="norm_small_layers"),
        # benchmark configuration 2: eight workers' gradients of 161 tensors
        _case("norm", 8, 25_557_032, 161, "f32", name="norm_8_workers"),
        # benchmark configuration 4's length, a worker's bf16 gradients
        _case("norm", 1, 355_000_000, 290, "bf16", name="norm_bf16_large"),
        # fp16 gradients of odd sizes that start anywhere in their bucket
        _case("clip", 1, 7_000_003, 61, "f16", odd=True, name="clip_f16_odd"),
        # benchmark configuration 3's length, bf16 matrices and fp32 vectors
        _case("clip", 1, 138_357_544, 32, "mixed", name="clip_mixed"),
        # benchmark configuration 1: four workers, one block each
        _case("gather", 4, 65_536, 6, "f32", name="gather_small"),
        # benchmark configuration 2, the way into bench.py's round
        _case("gather", 8, 25_557_032, 161, "f32", name="gather_8_workers"),
        # training with error feedback: bf16 gradients, fp32 vectors with the residual
        _case("gather", 4, 7_000_003, 61, "bf16", feedback=True, name="gather_feedback"),
        # a bucket's average back to bf16 gradients, below the norm that would be clipped
        _case("scatter", 1, 1_500_007, 20, "bf16", max_norm=1e4, name="scatter_bucket"),
        # benchmark configuration 4's length, to bf16 gradients
        _case("scatter", 1, 355_000_000, 290, "bf16", name="scatter_large"),
        # fp32 weights of a small model
        _case("adamw", 1, 65_536, 6, "f32", name="adamw_small"),
        # benchmark configuration 3's length: bf16 weights, fp32 master weights and moments
        _case("adamw", 1, 138_357_544, 32, "bf16", name="adamw_bf16_large"),
    ]


def draw(rng):
    """A case of the same ranges: a thousand to 2^28 elements over all workers (2^26.5 for the Adam step), up to 300
    tensors a worker and 16 workers, every type, tensors that start anywhere."""
    kind = rng.choice(["norm", "clip", "gather", "gather", "scatter", "adamw"])
    n = max(1, round(2 ** rng.uniform(0.0, 4.0))) if kind in ("norm", "clip", "gather") and rng.random() < 0.5 else 1
    d = int(2 ** rng.uniform(10.0, (26.5 if kind == "adamw" else 28.0) - math.log2(n))) + rng.randrange(0, 97)
    count = min(round(2 ** rng.uniform(0.0, 8.2)), d // 16)
    dtype = rng.choice(["f32", "bf16", "f16", "mixed"])
    feedback = kind == "gather" and rng.random() < 0.4
    flat = "bf16" if kind == "gather" and not feedback and rng.random() < 0.3 else "f32"
    return _case(kind, n, d, count, dtype, max_norm=rng.choice([0.25, 1.0, 1e4]), odd=rng.random() < 0.25, flat=flat, feedback=feedback)


def _sizes(case):
    """Sizes of a worker's tensors: proportional to lognormal(0, 1.5), d elements in all."""
    share = np.random.RandomState(case["d"] % 1_000_003).lognormal(0.0, 1.5, case["count"])
    at = np.floor(np.cumsum(share) / share.sum() * (case["d"] - case["count"])).astype(np.int64)
    at[-1] = case["d"] - case["count"]
    return (np.diff(at, prepend=0) + 1).tolist()


def _types(case, sizes):
    """The type of each tensor: of a mixed list the matrices are bf16, the smaller half is fp32."""
    if case["dtype"] != "mixed":
        return [TYPES[case["dtype"]]] * len(sizes)
    middle = sorted(sizes)[len(sizes) // 2]
    return [torch.float32 if s < middle else torch.bfloat16 for s in sizes]


def _up(v):
    return -(-v // ALIGN) * ALIGN


def _offsets(sizes):
    ends = np.cumsum([_up(s) for s in sizes]).tolist()
    return [0] + ends[:-1], ends[-1]


def _bucket(sizes, types, odd, device):
    """One zeroed allocation per type, and the tensors as pieces of them."""
    length, place = {}, []
    for i, (s, t) in enumerate(zip(sizes, types)):
        at = _up(length.get(t, 0)) + (1 + i % 7 if odd else 0)
        place.append(at)
        length[t] = at + s
    room = {t: torch.zeros(_up(v), dtype=t, device=device) for t, v in length.items()}
    return room, [room[t][at: at + s] for s, t, at in zip(sizes, types, place)]


def _fill(tensors, spread, gen):
    for x, s in zip(tensors, spread):
        x.normal_(0.0, float(s), generator=gen)


def prepare(case, seed):
    device = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    kind, n = case["kind"], case["n"]
    sizes = _sizes(case)
    types = _types(case, sizes)
    offsets, flat_length = _offsets(sizes)
    f32 = dict(dtype=torch.float32, device=device)
    state = {"case": case, "sizes": sizes, "offsets": offsets}
    # each tensor has a scale of its own, as layers have
    spread = np.exp(np.random.RandomState(seed % (1 << 31)).normal(math.log(1e-3), 1.0, len(sizes)))
    buckets = [_bucket(sizes, types, case["odd"], device) for _ in range(n)]
    state["rooms"] = [room for room, _ in buckets]
    tensors = state["tensors"] = [pieces for _, pieces in buckets]
    if kind in ("norm", "clip", "gather"):
        for pieces in tensors:
            _fill(pieces, spread, gen)
    if kind == "clip":
        buckets = [_bucket(sizes, types, case["odd"], device) for _ in range(n)]
        state["out_rooms"] = [room for room, _ in buckets]
        state["outs"] = [pieces for _, pieces in buckets]
    if kind == "gather":
        state["flats"] = torch.zeros(n, flat_length, dtype=TYPES[case["flat"]], device=device)
        if case["feedback"]:
            state["residuals"] = torch.zeros(n, flat_length, **f32)
            for row in state["residuals"]:
                _fill([row[o: o + s] for o, s in zip(offsets, sizes)], 0.1 * spread, gen)
    if kind in ("scatter", "adamw"):
        # decompression leaves its noise between the tensors too
        flat = state["flat"] = torch.empty(flat_length, **f32).normal_(0.0, 1e-4, generator=gen)
        _fill([flat[o: o + s] for o, s in zip(offsets, sizes)], spread, gen)
        inside = state["inside"] = torch.zeros(flat_length, dtype=torch.bool, device=device)
        for o, s in zip(offsets, sizes):
            inside[o: o + s] = True
    if kind == "adamw":
        state["moment1"] = torch.empty(flat_length, **f32).normal_(0.0, 1e-4, generator=gen) * inside
        state["moment2"] = torch.empty(flat_length, **f32).normal_(0.0, 1e-3, generator=gen).square() * inside
        _fill(tensors[0], np.full(len(sizes), 0.02), gen)
        state["master"] = None
        if case["dtype"] != "f32":
            master = state["master"] = torch.zeros(flat_length, **f32)
            for x, o, s in zip(tensors[0], offsets, sizes):
                master[o: o + s] = x
                master[o: o + s] *= 1.001
        # small tensors (biases, normalisation) take no weight decay
        middle = sorted(sizes)[len(sizes) // 2]
        state["decay"] = torch.tensor([0.0 if s < middle else DECAY for s in sizes], **f32)
        state["lr"] = torch.full((1,), 3e-4, **f32)
        state["step"] = torch.full((1,), 10 + seed % 5, dtype=torch.int64, device=device)
    if own:
        from paper_2302_08545_b200 import runner, thc, workloads
        w = workloads.Workload("plain", n=n, d=flat_length, log2_block=12, bits=4, granularity=30, table=workloads.TABLES[(4, 30)],
                               in_dtype=case["flat"], data_seed=0)
        ctx = state["ctx"] = runner.context_for(w)
        state["list"] = thc.Tensors(ctx, tensors)
        state["norms"] = torch.zeros(n, **f32)
        state["workspace"] = torch.empty(state["list"].workspace_bytes, dtype=torch.uint8, device=device)
        if kind == "clip":
            state["out_list"] = thc.Tensors(ctx, state["outs"])
    return state


def _norms(vectors):
    return torch.stack([v.float().square().sum(dtype=torch.float64).sqrt() for v in vectors])


def _factors(norms, case):
    return (case["max_norm"] / (norms + 1e-6)).clamp(max=1.0)


def _run_plain(state):
    case, kind, tensors = state["case"], state["case"]["kind"], state["tensors"]
    if kind in ("norm", "clip", "gather"):
        joined = [torch.cat(pieces) for pieces in tensors]
        norms = _norms(joined)
        if kind == "norm":
            return {"norms": norms.float()}
        c = _factors(norms, case).float()
        clipped = [v.float() * c[i] for i, v in enumerate(joined)]
        if kind == "clip":
            [[o.copy_(v) for o, v in zip(outs, flat.split(state["sizes"]))] for outs, flat in zip(state["outs"], clipped)]
            return {"norms": norms.float(), "outs": [list(room.values()) for room in state["out_rooms"]]}
        [[row[o: o + s].copy_(v) for v, o, s in zip(flat.split(state["sizes"]), state["offsets"], state["sizes"])]
         for row, flat in zip(state["flats"], clipped)]
        if case["feedback"]:
            state["flats"].add_(state["residuals"])
        return {"norms": norms.float(), "flats": state["flats"]}
    grad = state["flat"] * state["inside"]
    norms = _norms([grad])
    grad = grad * _factors(norms, case).float()
    if kind == "scatter":
        [x.copy_(grad[o: o + s]) for x, o, s in zip(tensors[0], state["offsets"], state["sizes"])]
        return {"norms": norms.float(), "tensors": list(state["rooms"][0].values())}
    t = state["step"].add_(1)
    m = state["moment1"].mul_(BETA1).add_(grad * (1 - BETA1))
    v = state["moment2"].mul_(BETA2).add_(grad * grad * (1 - BETA2))
    # 1 - beta^t in 64 bits
    by1, by2 = ((1 - torch.pow(torch.tensor(b, dtype=torch.float64, device=t.device), t)).float() for b in (BETA1, BETA2))
    move = state["lr"] * (m / by1) / ((v / by2).sqrt() + EPS)
    weights = tensors[0] if state["master"] is None else [state["master"][o: o + s] for o, s in zip(state["offsets"], state["sizes"])]
    keep = 1 - state["lr"] * state["decay"]
    [w.mul_(keep[i]).sub_(move[o: o + s]) for i, (w, o, s) in enumerate(zip(weights, state["offsets"], state["sizes"]))]
    if state["master"] is not None:
        [x.copy_(w) for x, w in zip(tensors[0], weights)]
    return _adamw_outputs(state, norms.float())


def _adamw_outputs(state, norms):
    out = {"norms": norms, "step": state["step"], "moment1": state["moment1"], "moment2": state["moment2"],
           "tensors": list(state["rooms"][0].values())}
    if state["master"] is not None:
        out["master"] = state["master"]
    return out


def _run_own(state):
    case, kind, ctx = state["case"], state["case"]["kind"], state["ctx"]
    norms, workspace, tensors = state["norms"], state["workspace"], state["list"]
    if kind == "norm":
        ctx.grad_norm(tensors, norms, workspace)
        return {"norms": norms}
    if kind == "clip":
        ctx.clip_grads(tensors, case["max_norm"], norms, workspace, out=state["out_list"])
        return {"norms": norms, "outs": [list(room.values()) for room in state["out_rooms"]]}
    if kind == "gather":
        residuals = list(state["residuals"]) if case["feedback"] else None
        ctx.gather_grads(tensors, case["max_norm"], list(state["flats"]), norms, workspace, ef=residuals)
        return {"norms": norms, "flats": state["flats"]}
    if kind == "scatter":
        ctx.scatter_grads(state["flat"], case["max_norm"], tensors, norms, workspace)
        return {"norms": norms, "tensors": list(state["rooms"][0].values())}
    ctx.adamw(state["flat"], tensors, state["lr"], state["step"], state["moment1"], state["moment2"], norms, workspace,
              master=state["master"], decay=state["decay"], betas=(BETA1, BETA2), eps=EPS, max_norm=case["max_norm"])
    return _adamw_outputs(state, norms)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    sizes = _sizes(case)
    per = [t.itemsize for t in _types(case, sizes)]
    n, d = case["n"], sum(sizes)
    tensors = n * sum(s * e for s, e in zip(sizes, per))
    kind = case["kind"]
    if kind == "norm":
        return {"bytes": tensors + 4 * n, "flops": 2 * n * d}
    if kind == "clip":
        return {"bytes": 2 * tensors + 4 * n, "flops": 3 * n * d}
    if kind == "gather":
        flat = n * _offsets(sizes)[1]
        return {"bytes": tensors + flat * TYPES[case["flat"]].itemsize + (4 * flat if case["feedback"] else 0) + 4 * n,
                "flops": (4 if case["feedback"] else 3) * n * d}
    if kind == "scatter":
        return {"bytes": 4 * d + tensors + 4, "flops": 3 * d}
    # moments read and written; the weights, with master weights also the tensors rounded from them
    weights = 2 * tensors if case["dtype"] == "f32" else 8 * d + tensors
    return {"bytes": 4 * d + 16 * d + weights, "flops": 20 * d}


def exact(case, seed):
    """The definitions in 64 bits, tensor by tensor."""
    state = prepare(case, seed)
    kind, tensors, places = case["kind"], state["tensors"], list(zip(state["offsets"], state["sizes"]))

    def length(pieces):
        return math.sqrt(math.fsum(float((x.double() ** 2).sum()) for x in pieces))

    def factor(norm):
        return min(1.0, case["max_norm"] / (norm + 1e-6))

    def on(device_of, values):
        return torch.tensor(values, dtype=torch.float64, device=device_of.device)

    def wide(room, pieces, values):
        """64-bit values of `pieces`, at their places in copies of their allocations."""
        copies = {t: r.double() for t, r in room.items()}
        for x, v in zip(pieces, values):
            copies[x.dtype][x.storage_offset(): x.storage_offset() + x.numel()] = v
        return list(copies.values())

    if kind in ("norm", "clip", "gather"):
        norms = [length(pieces) for pieces in tensors]
        out = {"norms": on(tensors[0][0], norms)}
        if kind == "clip":
            out["outs"] = [wide(room, outs, [x.double() * factor(norm) for x in pieces])
                           for room, outs, pieces, norm in zip(state["out_rooms"], state["outs"], tensors, norms)]
        if kind == "gather":
            flats = out["flats"] = torch.zeros(state["flats"].shape, dtype=torch.float64, device=tensors[0][0].device)
            for i, (pieces, norm) in enumerate(zip(tensors, norms)):
                for x, (o, s) in zip(pieces, places):
                    flats[i, o: o + s] = x.double() * factor(norm)
                    if case["feedback"]:
                        flats[i, o: o + s] += state["residuals"][i, o: o + s].double()
        return out
    grads = [state["flat"][o: o + s].double() for o, s in places]
    norm = length(grads)
    grads = [g * factor(norm) for g in grads]
    out = {"norms": on(state["flat"], [norm])}
    if kind == "scatter":
        out["tensors"] = wide(state["rooms"][0], tensors[0], grads)
        return out
    t = int(state["step"]) + 1
    lr = float(state["lr"])
    decay = state["decay"].tolist()
    moment1, moment2 = state["moment1"].double(), state["moment2"].double()
    master = None if state["master"] is None else state["master"].double()
    values = []
    for i, (g, (o, s)) in enumerate(zip(grads, places)):
        m, v = moment1[o: o + s], moment2[o: o + s]
        m.copy_(BETA1 * m + (1 - BETA1) * g)
        v.copy_(BETA2 * v + (1 - BETA2) * g * g)
        w = tensors[0][i].double() if master is None else master[o: o + s]
        w = w * (1 - lr * decay[i]) - lr * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
        values.append(w)
        if master is not None:
            master[o: o + s] = w
    out.update(step=state["step"] + 1, moment1=moment1, moment2=moment2, tensors=wide(state["rooms"][0], tensors[0], values))
    if master is not None:
        out["master"] = master
    return out
