"""The operators of a recurrent block that trains over whole unrolls, as cases that can be timed and compared.

  recurrence       h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(gate) ("blend"), or h_t = gate_t h_{t-1} + x_t
                   ("decay"): all steps of a batch of sequences, a single token as one step with its state
  recurrence_grad  its backward pass: gradients of gate, x and the first state
  block_norm       the join of a block with the residual stream: y = residual + scale act(gate) norm(x), and
                   norm(y), which the next block reads
  block_norm_grad  its backward pass, with the reductions of the parameters' gradients over all rows
  clip             the 2-norm over all gradients of a model, and the gradients scaled to a largest norm

Shapes are those of `inputs.py`, of the tests and of perf/operators.py, and generic ones around them: hidden sizes 300 to
1500, unrolls of 35 steps, batches 1 to 256, vocabularies up to 42000, sequences of up to 32768 steps.
`own` chooses who computes: elementary torch operations in 32 bits, or the library's entry points.
"""
import math

import torch

own = False

NORM_EPS = 1e-5
STATE_STEPS = 128                      # the forward pass leaves the state in front of every 128th step for the backward pass
DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
MOST = 1 << 25                         # entries of the largest cases but clip's
MOST_GRADS = 94_500_000                # entries of all gradients of the largest model


def listed():
    return [
        # One token of one sequence during generation (1024 units), its state handed on in full precision.  The smallest call.
        dict(name="recurrence_f32_1x1x1024", kind="recurrence", mode="blend", dtype="float32", steps=1, batch=1, n=1024,
             joined=False, ragged=False),
        # The medium model's unroll (35 steps of 20 sequences, 650 units), gate and candidate as one projection left them.
        dict(name="recurrence_f16_35x20x650", kind="recurrence", mode="blend", dtype="float16", steps=35, batch=20, n=650,
             joined=True, ragged=False),
        # One long document: few channels, so that time has to be split.
        dict(name="recurrence_bf16_32768x1x1024", kind="recurrence", mode="blend", dtype="bfloat16", steps=32768, batch=1,
             n=1024, joined=True, ragged=False),
        # Backward through the large model's unroll: 35 steps of 256 sequences.
        dict(name="recurrence_grad_bf16_35x256x1024", kind="recurrence_grad", mode="blend", dtype="bfloat16", steps=35,
             batch=256, n=1024, joined=True, ragged=False),
        # Backward through a padded batch of long sequences of unlike lengths, full precision, decay factors given, 300 units.
        dict(name="recurrence_grad_f32_4001x7x300", kind="recurrence_grad", mode="decay", dtype="float32", steps=4001, batch=7,
             n=300, joined=False, ragged=True),
        # One step of 64 sequences during generation: few rows.
        dict(name="block_norm_bf16_64x1024", kind="block_norm", dtype="bfloat16", residual="bfloat16", params="float32", rows=64,
             n=1024, gate="silu", scale=True),
        # All hidden states of 35 steps of 256 sequences, half precision.
        dict(name="block_norm_f16_8960x1024", kind="block_norm", dtype="float16", residual="float16", params="float32", rows=8960,
             n=1024, gate="sigmoid", scale=True),
        # Training, 1500 units: a full-precision residual stream, rows that do not begin on 16-byte boundaries.
        dict(name="block_norm_grad_bf16_8960x1500", kind="block_norm_grad", dtype="bfloat16", residual="float32", params="float32",
             rows=8960, n=1500, gate="silu", scale=True),
        # The medium model's unroll in full precision, without a gate.
        dict(name="block_norm_grad_f32_700x650", kind="block_norm_grad", dtype="float32", residual="float32", params="float32",
             rows=700, n=650, gate="none", scale=True),
        # The residual block on 300 units: six tensors, full precision.
        dict(name="clip_f32_300x1x0", kind="clip", dtype="float32", units=300, layers=1, vocab=0, tight=True),
        # Ten layers of 650 units, bfloat16 matrices with full-precision vectors: many tensors.
        dict(name="clip_bf16_650x10x10000", kind="clip", dtype="bfloat16", units=650, layers=10, vocab=10000, tight=True),
        # The large model with its vocabulary of 42000, full precision.  The largest case.
        dict(name="clip_f32_1024x1x42000", kind="clip", dtype="float32", units=1024, layers=1, vocab=42000, tight=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["recurrence", "recurrence_grad", "block_norm", "block_norm_grad", "clip"])
    dtype = rng.choice(["float32", "bfloat16", "float16"])
    if kind in ("recurrence", "recurrence_grad"):
        n = _log(rng, 64, 4096)
        batch = _log(rng, 1, 256)
        most = MOST // 2 if dtype == "float32" or kind == "recurrence_grad" else MOST
        steps = _log(rng, 1, max(1, min(32768, most // (n * batch))))
        return dict(kind=kind, mode=rng.choice(["blend", "decay"]), dtype=dtype, steps=steps, batch=batch, n=n,
                    joined=rng.random() < 0.5, ragged=rng.random() < 0.3)
    if kind in ("block_norm", "block_norm_grad"):
        n = _log(rng, 64, 8192)
        rows = _log(rng, 1, min(35840, (1 << 24) // n))
        return dict(kind=kind, dtype=dtype, residual=rng.choice(["float32", dtype]), params=rng.choice(["float32", dtype]), rows=rows,
                    n=n, gate=rng.choice(["none", "sigmoid", "silu"]), scale=rng.random() < 0.75)
    while True:
        case = dict(kind=kind, dtype=dtype, units=_log(rng, 64, 2048), layers=_log(rng, 1, 10), vocab=rng.choice([0, _log(rng, 64, 42000)]),
                    tight=rng.random() < 0.75)
        if sum(math.prod(shape) for shape, _ in _gradients(case)) <= MOST_GRADS:
            return case


def _gradients(case):
    """(shape, is a vector) of every gradient of a model of `layers` blocks, with its embedding and output layer."""
    u, v = case["units"], case["vocab"]
    shapes = []
    for _ in range(case["layers"]):
        shapes += [(4 * u, u), (u, 4 * u), (4 * u,), (u,), (u,), (u,)]
    if v:
        shapes += [(v, u), (v, u), (v,)]
    return [(s, len(s) == 1) for s in shapes]


def _lengths(case, g):
    """Lengths of a padded batch: spread evenly from none to all steps, in an order that the seed makes."""
    b = case["batch"]
    spread = torch.linspace(0 if b > 2 else case["steps"] // 2, case["steps"], b, device="cuda").round().long()
    return spread[torch.randperm(b, generator=g, device="cuda")]


def _spread_total(case):
    """The sum of those lengths."""
    b, t = case["batch"], case["steps"]
    lo = 0 if b > 2 else t // 2
    return sum(int(round(lo + (t - lo) * (i / (b - 1)))) for i in range(b)) if b > 1 else lo


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda") * scale

    s = {"case": case}
    if case["kind"] in ("recurrence", "recurrence_grad"):
        steps, batch, n = case["steps"], case["batch"], case["n"]
        # units that forget within a few steps and units that hold for hundreds
        gate = normal(steps, batch, n) + torch.rand(n, generator=g, device="cuda") * 6 - 1
        x = normal(steps, batch, n)
        if case["mode"] == "decay":
            gate = torch.sigmoid(gate)
            x = x * (1 - gate)
        s["lengths"] = None
        if case["ragged"]:
            s["lengths"] = _lengths(case, g)
            # whatever an earlier batch left in the padding
            behind = torch.arange(steps, device="cuda")[:, None] >= s["lengths"]
            gate, x = (v.masked_fill(behind[:, :, None], math.nan) for v in (gate, x))
        if case["joined"]:
            both = torch.cat([gate, x], 2).to(dt)
            s["gate"], s["x"] = both[:, :, :n], both[:, :, n:]
        else:
            s["gate"], s["x"] = gate.to(dt), x.to(dt)
        s["h0"] = normal(batch, n, scale=0.5)
        if case["kind"] == "recurrence_grad":
            s["dhs"] = normal(steps, batch, n, scale=1.0 / (steps * batch)).to(dt)
            s["dh_last"] = normal(batch, n, scale=1.0 / batch)
            # what the forward pass left: the states in front of steps 128, 256, ...
            s["states"] = None
            if steps > STATE_STEPS:
                keep, add, _ = _factors(s["gate"], s["x"], case["mode"], s["lengths"])
                s["states"] = _scan(keep, add, s["h0"])[STATE_STEPS - 1:steps - 1:STATE_STEPS].contiguous()
    elif case["kind"] in ("block_norm", "block_norm_grad"):
        rows, n, rt, pt = case["rows"], case["n"], DTYPES[case["residual"]], DTYPES[case["params"]]
        # a block's output: units of unlike scale, and a mean that is not zero
        s["x"] = (normal(rows, n) * (0.5 + normal(n).abs()) + 0.25).to(dt)
        s["residual"] = normal(rows, n).to(rt)
        s["gate"] = normal(rows, n).to(dt) if case["gate"] != "none" else None
        for key in ("weight", "next_weight"):
            s[key] = (1 + normal(n, scale=0.1)).to(pt)
        for key in ("bias", "next_bias"):
            s[key] = normal(n, scale=0.1).to(pt)
        s["scale"] = (0.5 + normal(n, scale=0.1)).to(pt) if case["scale"] else None
        if case["kind"] == "block_norm_grad":
            y, _, s["stats"] = _plain_block_norm(s, case)
            s["y"] = y.to(rt)
            del s["residual"]
            s["dy"] = normal(rows, n, scale=1.0 / rows).to(rt)
            s["dnormed"] = normal(rows, n, scale=1.0 / rows).to(dt)
    else:
        s["grads"] = [normal(*shape, scale=1e-3).to(torch.float32 if vector else dt) for shape, vector in _gradients(case)]
        s["out"] = [torch.empty_like(t) for t in s["grads"]]
        entries = sum(t.numel() for t in s["grads"])
        # the expected norm, and a limit that halves it or lets it through
        s["max_norm"] = 1e-3 * entries ** 0.5 * (0.5 if case["tight"] else 2.0)
    return s


def _factors(gate, x, mode, lengths):
    """What is kept of the state, what is added to it, and 1 - kept; padding keeps the state."""
    gate, x = gate.float(), x.float()
    if mode == "blend":
        keep, take = 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))
        add = take * x
    else:
        keep, take, add = gate, None, x
    if lengths is not None:
        behind = _behind(gate, lengths)
        keep, add = keep.masked_fill(behind, 1.0), add.masked_fill(behind, 0.0)
        take = None if take is None else take.masked_fill(behind, 0.0)
    return keep, add, take


def _behind(t, lengths):
    return (torch.arange(t.shape[0], device=t.device)[:, None] >= lengths)[:, :, None]


def _scan(keep, add, h):
    """h_t = keep_t h_{t-1} + add_t for all steps: spans of 1, 2, 4, ... steps are joined."""
    add = torch.cat([add[:1] + keep[:1] * h, add[1:]])
    d = 1
    while d < add.shape[0]:
        add = torch.cat([add[:d], add[d:] + keep[d:] * add[:-d]])
        keep = torch.cat([keep[:d], keep[d:] * keep[:-d]])
        d *= 2
    return add


def _plain_recurrence(s, case):
    keep, add, _ = _factors(s["gate"], s["x"], case["mode"], s["lengths"])
    hs = _scan(keep, add, s["h0"])
    last = hs[-1].clone()
    if s["lengths"] is not None:
        hs = hs.masked_fill(_behind(hs, s["lengths"]), 0.0)
    return hs, last


def _plain_recurrence_grad(s, case):
    keep, add, take = _factors(s["gate"], s["x"], case["mode"], s["lengths"])
    hs = _scan(keep, add, s["h0"])
    before = torch.cat([s["h0"][None], hs[:-1]])
    d = s["dhs"].float()
    behind = None
    if s["lengths"] is not None:
        behind = _behind(d, s["lengths"])
        d = d.masked_fill(behind, 0.0)
    after = torch.cat([keep[1:], torch.ones_like(keep[:1])])
    e = _scan(after.flip(0), d.flip(0), s["dh_last"]).flip(0)
    if case["mode"] == "blend":
        x = s["x"].float()
        x = x if behind is None else x.masked_fill(behind, 0.0)
        dgate, dx = e * (before - x) * keep * take, e * take
    else:
        dgate, dx = e * before, e
    if behind is not None:
        dgate, dx = dgate.masked_fill(behind, 0.0), dx.masked_fill(behind, 0.0)
    return dgate, dx, keep[0] * e[0]


def _gate(s, kind):
    """act(gate) and its slope; 1 and 0 without a gate."""
    if kind == "none":
        return 1.0, 0.0
    z = s["gate"].float()
    p = 1 / (1 + torch.exp(-z))
    if kind == "sigmoid":
        return p, p * (1 - p)
    return z * p, p * (1 + z * (1 - p))


def _centred(x, mean=None, rstd=None):
    """(x - mean) rstd, with the rows' own mean and rstd where none are given."""
    if mean is None:
        mean = x.sum(1) / x.shape[1]
        d = x - mean[:, None]
        rstd = 1 / torch.sqrt((d * d).sum(1) / x.shape[1] + NORM_EPS)
    return (x - mean[:, None]) * rstd[:, None], mean, rstd


def _plain_block_norm(s, case):
    z, mean, rstd = _centred(s["x"].float())
    u = z * s["weight"].float() + s["bias"].float()
    if s["scale"] is not None:
        u = u * s["scale"].float()
    y = s["residual"].float() + u * _gate(s, case["gate"])[0]
    z, mean_y, rstd_y = _centred(y)
    return y, z * s["next_weight"].float() + s["next_bias"].float(), torch.stack([mean, rstd, mean_y, rstd_y])


def _norm_slope(g, z, rstd):
    """The gradient of a row in front of (x - mean) rstd = z, given that behind it."""
    n = z.shape[1]
    return rstd[:, None] * (g - g.sum(1, keepdim=True) / n - z * ((g * z).sum(1, keepdim=True) / n))


def _plain_block_norm_grad(s, case):
    stats = s["stats"]
    z, _, _ = _centred(s["x"].float(), stats[0], stats[1])
    zy, _, _ = _centred(s["y"].float(), stats[2], stats[3])
    dn = s["dnormed"].float()
    dy = s["dy"].float() + _norm_slope(dn * s["next_weight"].float(), zy, stats[3])
    u = z * s["weight"].float() + s["bias"].float()
    a, slope = _gate(s, case["gate"])
    scaled = dy if s["scale"] is None else dy * s["scale"].float()
    du = scaled * a
    out = {"dx": _norm_slope(du * s["weight"].float(), z, stats[1]), "dresidual": dy, "dweight": (du * z).sum(0), "dbias": du.sum(0),
           "dnext_weight": (dn * zy).sum(0), "dnext_bias": dn.sum(0)}
    if case["gate"] != "none":
        out["dgate"] = scaled * u * slope
    if s["scale"] is not None:
        out["dscale"] = (dy * a * u).sum(0)
    return out


def _types(case):
    """The type of each result of block_norm_grad."""
    dt, rt, pt = (DTYPES[case[key]] for key in ("dtype", "residual", "params"))
    return {"dx": dt, "dgate": dt, "dresidual": rt, "dweight": pt, "dbias": pt, "dscale": pt, "dnext_weight": pt, "dnext_bias": pt}


def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "recurrence":
        hs, last = _plain_recurrence(state, case)
        return {"hs": hs.to(dt), "h_last": last}
    if case["kind"] == "recurrence_grad":
        dgate, dx, dh0 = _plain_recurrence_grad(state, case)
        return {"dgate": dgate.to(dt), "dx": dx.to(dt), "dh0": dh0}
    if case["kind"] == "block_norm":
        y, normed, stats = _plain_block_norm(state, case)
        return {"y": y.to(DTYPES[case["residual"]]), "normed": normed.to(dt), "stats": stats}
    if case["kind"] == "block_norm_grad":
        types = _types(case)
        return {key: v.to(types[key]) for key, v in _plain_block_norm_grad(state, case).items()}
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for t in state["grads"]:
        t = t.float()
        total = total + (t * t).sum().double()
    norm = total.sqrt()
    c = torch.clamp(state["max_norm"] / norm, max=1.0).float()
    for t, o in zip(state["grads"], state["out"]):
        o.copy_(t.float() * c)
    return {"norm": norm.float(), "grads": state["out"]}


def _own(state, case):
    import paper_1802_00150_amd as amq
    if case["kind"] == "recurrence":
        hs, last, _ = amq.linear_recurrence(state["gate"], state["x"], state["h0"], mode=case["mode"], lengths=state["lengths"])
        return {"hs": hs, "h_last": last}
    if case["kind"] == "recurrence_grad":
        dgate, dx, dh0 = amq.linear_recurrence_backward(state["dhs"], state["gate"], state["x"], state["h0"], state["states"],
                                                        dh_last=state["dh_last"], mode=case["mode"], lengths=state["lengths"])
        return {"dgate": dgate, "dx": dx, "dh0": dh0}
    if case["kind"] == "block_norm":
        y, normed, stats = amq.block_norm(state["x"], state["residual"], state["weight"], state["bias"], gate=state["gate"],
                                          activation=case["gate"], scale=state["scale"], next_weight=state["next_weight"],
                                          next_bias=state["next_bias"], eps=NORM_EPS)
        return {"y": y, "normed": normed, "stats": stats}
    if case["kind"] == "block_norm_grad":
        results = amq.block_norm_backward(state["dy"], state["dnormed"], state["x"], state["y"], state["stats"], state["weight"],
                                          state["bias"], gate=state["gate"], activation=case["gate"], scale=state["scale"],
                                          next_weight=state["next_weight"], next_bias=state["next_bias"])
        keys = ("dx", "dresidual", "dgate", "dweight", "dbias", "dscale", "dnext_weight", "dnext_bias")
        return {key: v for key, v in zip(keys, results) if v is not None}
    norm = amq.clip_gradients(state["grads"], state["max_norm"], out=state["out"])
    return {"norm": norm, "grads": state["out"]}


def work(case):
    size = {"float32": 4, "bfloat16": 2, "float16": 2}
    s = size[case["dtype"]]
    if case["kind"] in ("recurrence", "recurrence_grad"):
        width = case["batch"] * case["n"]
        # padding is written, not read
        entries = case["steps"] * width
        read = _spread_total(case) * case["n"] if case["ragged"] else entries
        if case["kind"] == "recurrence":
            return {"bytes": s * (2 * read + entries) + 8 * width, "flops": 10 * read}
        return {"bytes": s * (3 * read + 2 * entries) + 4 * width * (3 + (case["steps"] - 1) // STATE_STEPS), "flops": 25 * read}
    if case["kind"] in ("block_norm", "block_norm_grad"):
        rows, n, r, p = case["rows"], case["n"], size[case["residual"]], size[case["params"]]
        gate, scale = int(case["gate"] != "none"), int(case["scale"])
        if case["kind"] == "block_norm":
            return {"bytes": rows * n * (s * (2 + gate) + 2 * r) + n * p * (4 + scale) + 16 * rows, "flops": rows * n * 25}
        return {"bytes": rows * n * (s * (3 + 2 * gate) + 3 * r) + n * p * (3 + 4 + 2 * scale) + 16 * rows, "flops": rows * n * 50}
    entries = [(math.prod(shape), 4 if vector else s) for shape, vector in _gradients(case)]
    return {"bytes": 2 * sum(n * size for n, size in entries) + 4, "flops": 3 * sum(n for n, _ in entries)}


def exact(case, seed):
    """The definitions in binary64, on the same inputs: steps one after the other, gradients of the norms by autograd."""
    s = prepare(case, seed)
    v = {key: t.double() for key, t in s.items() if isinstance(t, torch.Tensor) and key != "lengths"}
    if case["kind"] in ("recurrence", "recurrence_grad"):
        return _exact_recurrence(case, v, s["lengths"])
    if case["kind"] == "block_norm":
        y, normed, stats = _exact_block_norm(case, v)
        return {"y": y, "normed": normed, "stats": stats}
    if case["kind"] == "block_norm_grad":
        return _exact_block_norm_grad(case, v)
    total = 0.0
    for t in s["grads"]:
        total = total + torch.linalg.vector_norm(t, dtype=torch.float64) ** 2
    norm = total ** 0.5
    c = s["max_norm"] / torch.maximum(norm, torch.full_like(norm, s["max_norm"]))
    return {"norm": norm, "grads": [torch.mul(t.double(), c) for t in s["grads"]]}


def _exact_recurrence(case, v, lengths):
    steps, blend = case["steps"], case["mode"] == "blend"
    h, hs = v["h0"], []
    for t in range(steps):
        x, g = v["x"][t], v["gate"][t]
        new = torch.lerp(x, h, torch.sigmoid(g)) if blend else torch.addcmul(x, g, h)
        if lengths is not None:
            new = torch.where((lengths > t)[:, None], new, h)
        hs.append(h)                   # in front of the step
        h = new
    if case["kind"] == "recurrence":
        out = torch.stack(hs[1:] + [h])
        if lengths is not None:
            out = torch.stack([torch.where((lengths > t)[:, None], out[t], torch.zeros_like(h)) for t in range(steps)])
        return {"hs": out, "h_last": h}
    e = v["dh_last"]
    dgate, dx = torch.empty_like(v["dhs"]), torch.empty_like(v["dhs"])
    for t in reversed(range(steps)):
        x, g = v["x"][t], v["gate"][t]
        total = e + v["dhs"][t]
        if blend:
            f = torch.sigmoid(g)
            forget = torch.sigmoid(-g)
            dg, d, new = total * (hs[t] - x) * f * forget, total * forget, total * f
        else:
            dg, d, new = total * hs[t], total, total * g
        if lengths is not None:
            here = (lengths > t)[:, None]
            dg, d = (torch.where(here, w, torch.zeros_like(w)) for w in (dg, d))
            new = torch.where(here, new, e)
        dgate[t], dx[t], e = dg, d, new
    return {"dgate": dgate, "dx": dx, "dh0": e}


def _exact_gate(case, gate):
    return torch.sigmoid(gate) if case["gate"] == "sigmoid" else torch.nn.functional.silu(gate)


def _exact_block_norm(case, v):
    n = case["n"]
    var, mean = torch.var_mean(v["x"], 1, unbiased=False)
    u = torch.addcmul(v["bias"], (v["x"] - mean.unsqueeze(1)) / (var + NORM_EPS).sqrt().unsqueeze(1), v["weight"])
    if "gate" in v:
        u = u * _exact_gate(case, v["gate"])
    y = v["residual"] + (u * v["scale"] if "scale" in v else u)
    normed = torch.nn.functional.layer_norm(y, (n,), v["next_weight"], v["next_bias"], NORM_EPS)
    var_y, mean_y = torch.var_mean(y, 1, unbiased=False)
    return y, normed, torch.stack([mean, (var + NORM_EPS).pow(-0.5), mean_y, (var_y + NORM_EPS).pow(-0.5)])


def _exact_block_norm_grad(case, v):
    # z as the saved statistics give it; through them the gradient goes by the formula of the layer norm
    n = case["n"]
    mean, rstd, mean_y, rstd_y = (t.unsqueeze(1) for t in v["stats"])
    z, zy = (v["x"] - mean) * rstd, (v["y"] - mean_y) * rstd_y

    def through(g, z, rstd):
        along = torch.einsum("rn,rn->r", g, z).unsqueeze(1)
        return (g * n - g.sum(1, keepdim=True) - z * along) * (rstd / n)

    dy = v["dy"] + through(v["dnormed"] * v["next_weight"], zy, rstd_y)
    leaves = {key: v[key].clone().requires_grad_() for key in ("weight", "bias", "scale", "gate") if key in v}
    leaf_z = z.clone().requires_grad_()
    u = torch.addcmul(leaves["bias"], leaf_z, leaves["weight"])
    if "gate" in leaves:
        u = u * _exact_gate(case, leaves["gate"])
    if "scale" in leaves:
        u = u * leaves["scale"]
    names = list(leaves)
    dz, *grads = torch.autograd.grad(u, [leaf_z] + [leaves[key] for key in names], dy)
    out = {"dx": through(dz, z, rstd), "dresidual": dy, "dnext_weight": torch.einsum("rn,rn->n", v["dnormed"], zy),
           "dnext_bias": v["dnormed"].sum(0)}
    out.update({"d" + key: t for key, t in zip(names, grads)})
    return out
