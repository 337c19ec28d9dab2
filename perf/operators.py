"""Three operators that stand around the matrix products of a population's training step, as a user calls them and in plain torch.

"clip"    the gradient norm of every member over all its tensors, and the gradients scaled down to the member's largest norm
"rotary"  rotary positions on query and key heads: two pair layouts, part of a head, frequencies scaled for long contexts, and the transposed
          rotation of the backward pass
"block"   the norm after a block, its gate, the scaled residual sum and the norm before the next block in one pass, and their gradients

`own` chooses between the library's kernels and the plain form; both take what `prepare` makes.  Sizes are those of the
repository's workloads (a transformer of width 512 with 4 blocks, 16 members of 32 sequences of 128 positions; the actor-critic and the small
classifier networks), single tokens, and generic large and odd ones.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}


def _transformer_tensors(d=512, f=2048, V=8192, S=128, blocks=4):
    """Element counts of the parameter arrays of one transformer of the repository's workload."""
    block = [d, d, d * 3 * d, 3 * d, d * d, d, d, d, d * f, f, f * d, d]
    return [V * d, S * d] + block * blocks + [d, d, d * V, V]


def _mlp_tensors(dims):
    out = []
    for a, b in zip(dims[:-1], dims[1:]):
        out += [a * b, b]
    return out


def _text(sizes):
    return "-".join(str(n) for n in sizes)


def listed():
    return [
        # ---- clip: gradients are read where backward left them and written to the buffer that the optimiser or an all-reduce takes
        # the small classifier population: 8 members, four tensors of 2372 values in all; latency
        dict(op="clip", name="clip_small_classifier", P=8, sizes=_text(_mlp_tensors([32, 64, 4])), dtype="fp32"),
        # the agents: 128 members of 202k parameters in six tensors, one chip-cache-sized gradient
        dict(op="clip", name="clip_agents", P=128, sizes=_text(_mlp_tensors([512, 256, 256, 19])), dtype="fp32"),
        # the language models: 16 members of 21 million parameters in 54 tensors, far more than the caches hold
        dict(op="clip", name="clip_transformers", P=16, sizes=_text(_transformer_tensors()), dtype="fp32"),
        # gradients kept in bf16, tensors of odd sizes and of one value
        dict(op="clip", name="clip_bf16_odd", P=3, sizes=_text([1000003, 77, 135201, 1, 4999999, 513]), dtype="bf16"),
        # ---- rotary
        # generation: the newest token of 16 sequences far into their contexts, 8 query and 8 key heads
        dict(op="rotary", name="rotary_single_token", rows=16, heads=16, width=64, rot=64, layout="half", scaling="none", dtype="bf16", far=32768,
             period=0, backward=False),
        # the training step of the transformer population: query and key parts of [65536][1536]
        dict(op="rotary", name="rotary_train", rows=65536, heads=16, width=64, rot=64, layout="half", scaling="none", dtype="bf16", far=128,
             period=128, backward=False),
        # its backward form in fp32 with sizes that fit nothing: half of each 84-wide head is rotated, pairs lie side by side
        dict(op="rotary", name="rotary_backward_odd", rows=9973, heads=5, width=84, rot=42, layout="interleaved", scaling="linear", dtype="fp32",
             far=1000000, period=0, backward=True),
        # a long context read at once: 131072 positions, 32 query and 8 key heads of 128, frequencies scaled by their wavelength
        dict(op="rotary", name="rotary_long_context", rows=131072, heads=40, width=128, rot=128, layout="interleaved", scaling="ramp", dtype="bf16",
             far=131072, period=0, backward=False),
        # ---- block
        # generation: one token of each of 4 sequences through a model of width 2048
        dict(op="block", name="block_single_token", P=1, rows=4, d=2048, post="rms", pre="rms", gate="none", act="none", dtype="bf16", res="bf16",
             train=False),
        # the forward pass of the transformer population, a learned gate per channel
        dict(op="block", name="block_forward", P=16, rows=4096, d=512, post="layer", pre="layer", gate="vector", act="none", dtype="bf16", res="bf16",
             train=False),
        # forward and backward of the same population, a sigmoid gate per token and channel, residual stream in fp32
        dict(op="block", name="block_train_gated", P=16, rows=4096, d=512, post="rms", pre="rms", gate="rows", act="sigmoid", dtype="bf16", res="fp32",
             train=True),
        # one wide model with an odd width and an odd number of rows
        dict(op="block", name="block_train_wide_odd", P=1, rows=8191, d=5001, post="rms", pre="layer", gate="vector", act="none", dtype="bf16",
             res="bf16", train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["clip", "rotary", "block"])
    if op == "clip":
        P = _log_int(rng, 1, 128)
        total = _log_int(rng, 100, 300_000_000 // P)     # per member
        n = _log_int(rng, 1, 120)
        cuts = [rng.random() ** 3 + 1e-4 for _ in range(n)]
        return dict(op="clip", P=P, sizes=_text([max(1, int(total * c / sum(cuts))) for c in cuts]), dtype=rng.choice(["fp32", "bf16"]))
    if op == "rotary":
        heads, width = _log_int(rng, 1, 40), 2 * rng.randint(4, 64)
        rot = width if rng.random() < 0.5 else 2 * rng.randint(2, width // 2)
        rows = _log_int(rng, 1, 131072)
        far = _log_int(rng, 64, 1 << 20)
        return dict(op="rotary", rows=rows, heads=heads, width=width, rot=rot, layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "base", "ramp"]), dtype=rng.choice(["fp32", "bf16"]) if rows * heads * width < 300_000_000 else "bf16",
                    far=far, period=far if rng.random() < 0.3 else 0, backward=rng.random() < 0.4)
    d = _log_int(rng, 8, 8192)
    if rng.random() < 0.6:
        d = max(8, d // 8 * 8)
    P = _log_int(rng, 1, 32)
    rows = _log_int(rng, 1, max(1, 32_000_000 // (d * P)))
    gate = rng.choice(["none", "vector", "rows"])
    post, pre = rng.choice([("layer", "layer"), ("rms", "rms"), ("rms", "layer"), ("layer", "rms"), ("none", "layer"), ("none", "rms"), ("rms", "none")])
    return dict(op="block", P=P, rows=rows, d=d, post=post, pre=pre, gate=gate, act="none" if gate == "none" else rng.choice(["none", "sigmoid", "silu", "tanh"]),
                dtype=rng.choice(["bf16", "bf16", "fp32"]), res=rng.choice(["bf16", "fp32"]), train=rng.random() < 0.6)


# ---- inputs ------------------------------------------------------------------------------------------------------------------------------------------

MAX_NORM = 1.0
BASE, GAIN = 10000.0, 1.0
FACTOR, TRAINED, LOW, HIGH, RAMP_GAIN = 8.0, 4096, 1.0, 32.0, 1.2   # a context eight times the trained one
EPS, ALPHA, BETA = 1e-5, 1.0, 0.7


def _inputs(case, seed):
    """The case's tensors: name -> tensor or list of tensors, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device="cuda").mul_(scale).to(dtype)

    if case["op"] == "clip":
        sizes = [int(n) for n in case["sizes"].split("-")]
        P, dt = case["P"], DTYPES[case["dtype"]]
        # members' norms spread over 0.2 to 5 around the largest one allowed: some are clipped, some are not
        norm = torch.exp(torch.empty(P, 1, device="cuda").uniform_(math.log(0.2), math.log(5.0), generator=g))
        scale = norm / math.sqrt(sum(sizes))
        return dict(grads=[(torch.randn(P, n, generator=g, device="cuda") * scale).to(dt) for n in sizes],
                    max_norm=torch.full((P,), MAX_NORM, device="cuda"))
    if case["op"] == "rotary":
        rows, heads, width, dt = case["rows"], case["heads"], case["width"], DTYPES[case["dtype"]]
        pos = None
        if not case["period"]:      # positions of a packed batch, any order
            pos = torch.randint(0, case["far"], (rows,), generator=g, device="cuda", dtype=torch.int32)
        # the rotated heads lie beside heads that are not (values), as in a joint projection's output
        return dict(x=normal(rows, heads + max(1, heads // 2), width, dtype=dt)[:, :heads], positions=pos)
    P, rows, d = case["P"], case["rows"], case["d"]
    dt, rt = DTYPES[case["dtype"]], DTYPES[case["res"]]
    n = P * rows
    s = dict(y=normal(n, d, scale=0.5, dtype=dt), x=normal(n, d, scale=2.0, dtype=rt))
    params = {}
    if case["post"] != "none":
        params["post_gain"] = 1.0 + normal(P, d, scale=0.1)
    if case["post"] == "layer":
        params["post_bias"] = normal(P, d, scale=0.1)
    if case["pre"] != "none":
        params["pre_gain"] = 1.0 + normal(P, d, scale=0.1)
    if case["pre"] == "layer":
        params["pre_bias"] = normal(P, d, scale=0.1)
    if case["gate"] == "vector":
        params["gate"] = 0.5 + normal(P, d, scale=0.2)
    s["params"] = params
    s["gate"] = normal(n, d, dtype=dt) if case["gate"] == "rows" else None
    if case["train"]:
        s["dout"] = normal(n, d, scale=1e-2, dtype=rt)
        s["dz"] = normal(n, d, scale=1e-2, dtype=dt) if case["pre"] != "none" else None
    return s


def _rope_settings(case):
    k = dict(base=BASE, layout=case["layout"], scaling=case["scaling"])
    if case["scaling"] != "none":
        k["factor"] = FACTOR
    if case["scaling"] == "ramp":
        k.update(trained=TRAINED, low=LOW, high=HIGH, gain=RAMP_GAIN)
    return k


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "clip":
        s["outs"] = [torch.empty_like(t) for t in s["grads"]]
    elif case["op"] == "rotary":
        s["out"] = torch.empty(case["rows"], case["heads"], case["width"], dtype=s["x"].dtype, device="cuda")
    if own:
        from paper_1711_09846_amd import binding
        if case["op"] == "clip":
            s["plan"] = binding.GradClip(s["grads"], s["outs"])
        elif case["op"] == "rotary":
            s["plan"] = binding.Rotary(case["rot"], **_rope_settings(case))
        else:
            s["plan"] = binding.BlockNorm(case["d"], members=case["P"], post=case["post"], pre=case["pre"], gate=case["gate"], act=case["act"],
                                          eps=EPS, alpha=ALPHA, beta=BETA)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    return {"clip": _clip, "rotary": _rotary, "block": _block}[case["op"]](state, case)


def _run_own(s, case):
    if case["op"] == "clip":
        norms = s["plan"](s["max_norm"])
        return dict(norms=norms, grads=s["outs"])
    if case["op"] == "rotary":
        return s["plan"](s["x"], s["out"], positions=s["positions"], period=case["period"], backward=case["backward"])
    out, z, stats = s["plan"].forward(s["y"], s["x"], s["params"], gate=s["gate"])
    res = dict(out=out) if z is None else dict(out=out, z=z)
    if case["train"]:
        dy, dx, dgate, grads = s["plan"].backward(s["y"], s["x"], s["params"], stats, s["dout"], s["dz"], gate=s["gate"])
        res.update(dy=dy, dx=dx, **{"d_" + k: v for k, v in grads.items()})
        if dgate is not None:
            res["dgate"] = dgate
    return res


def _clip(s, case):
    grads = s["grads"]
    sq = torch.zeros(case["P"], dtype=torch.float64, device="cuda")
    for t in grads:                                           # (long sums: in 64 bits)
        v = t.float()
        sq += (v * v).sum(dim=1, dtype=torch.float64)
    norms = sq.sqrt().float()
    c = torch.where(norms > s["max_norm"], s["max_norm"] / norms, torch.ones_like(norms))
    for t, o in zip(grads, s["outs"]):
        o.copy_(t.float() * c[:, None])
    return dict(norms=norms, grads=s["outs"])


def _frequencies(case):
    """Radians per position of every pair, 64 bits."""
    r = case["rot"]
    j = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    base = BASE
    if case["scaling"] == "base" and r > 2:
        base = BASE * FACTOR ** (r / (r - 2))
    f = base ** (-2.0 * j / r)
    if case["scaling"] == "linear":
        f = f / FACTOR
    if case["scaling"] == "ramp":
        w = ((TRAINED * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        f = f * (w + (1.0 - w) / FACTOR)
    return f


def _positions(s, case):
    if s["positions"] is not None:
        return s["positions"]
    return torch.arange(case["rows"], device="cuda") % case["period"]


def _rotary(s, case):
    r = case["rot"]
    angle = _positions(s, case).double()[:, None] * _frequencies(case)      # (far positions: in 64 bits)
    gain = RAMP_GAIN if case["scaling"] == "ramp" else GAIN
    cos, sin = (angle.cos() * gain).float()[:, None, :], (angle.sin() * gain).float()[:, None, :]
    if case["backward"]:
        sin = -sin
    x = s["x"].float()
    if case["layout"] == "half":
        a, b = x[..., : r // 2], x[..., r // 2 : r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    out = s["out"]
    out[..., :r] = turned.to(out.dtype)
    out[..., r:] = s["x"][..., r:]
    return out


def _norm(kind, v, gain, bias):
    """(normalised and scaled rows, the rows before gain and bias, 1 / spread)."""
    if kind == "none":
        return v, None, None
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    rstd = ((v * v).mean(-1, keepdim=True) + EPS).rsqrt()
    hat = v * rstd
    return hat * gain + (bias if bias is not None else 0.0), hat, rstd


def _norm_backward(kind, dv, gain, hat, rstd):
    if kind == "none":
        return dv
    w = dv * gain
    d = w - hat * (w * hat).mean(-1, keepdim=True)
    if kind == "layer":
        d = d - w.mean(-1, keepdim=True)
    return rstd * d


def _gate(act, g):
    """The gate's factor and its derivative."""
    if act == "none":
        return g, torch.ones_like(g)
    if act == "tanh":
        t = g.tanh()
        return t, 1.0 - t * t
    s = 1.0 / (1.0 + (-g).exp())
    if act == "sigmoid":
        return s, s * (1.0 - s)
    return g * s, s * (1.0 + g * (1.0 - s))


def _block(s, case):
    P, rows, d = case["P"], case["rows"], case["d"]
    p = {k: v[:, None, :] for k, v in s["params"].items()}
    rows_of = lambda t: t.float().view(P, rows, d)  # noqa: E731
    x = rows_of(s["x"])
    u, yhat, yr = _norm(case["post"], rows_of(s["y"]), p.get("post_gain"), p.get("post_bias"))
    factor = slope = None
    if case["gate"] != "none":
        factor, slope = _gate(case["act"], p["gate"] if case["gate"] == "vector" else rows_of(s["gate"]))
    out = ALPHA * x + BETA * (u if factor is None else factor * u)
    z, xhat, xr = _norm(case["pre"], out, p.get("pre_gain"), p.get("pre_bias"))
    flat = lambda t, like: t.to(like.dtype).view(P * rows, d)  # noqa: E731
    res = dict(out=flat(out, s["x"]))
    if case["pre"] != "none":
        res["z"] = flat(z, s["y"])
    if not case["train"]:
        return res
    t = rows_of(s["dout"])
    if case["pre"] != "none":
        dz = rows_of(s["dz"])
        t = t + _norm_backward(case["pre"], dz, p["pre_gain"], xhat, xr)
        res["d_pre_gain"] = (dz * xhat).sum(1)
        if "pre_bias" in p:
            res["d_pre_bias"] = dz.sum(1)
    res["dx"] = flat(ALPHA * t, s["x"])
    v = BETA * (t if factor is None else factor * t)
    if case["gate"] != "none":
        dgate = BETA * slope * u * t
        if case["gate"] == "vector":
            res["d_gate"] = dgate.sum(1)
        else:
            res["dgate"] = flat(dgate, s["y"])
    if case["post"] != "none":
        res["d_post_gain"] = (v * yhat).sum(1)
        if "post_bias" in p:
            res["d_post_bias"] = v.sum(1)
    res["dy"] = flat(_norm_backward(case["post"], v, p.get("post_gain"), yhat, yr), s["y"])
    return res


# ---- the same in 64 bits, from the definitions ----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "clip":
        norms = torch.stack([torch.linalg.vector_norm(t.double(), dim=1) for t in s["grads"]]).pow(2).sum(0).sqrt()
        shrink = (s["max_norm"].double() / norms).clamp(max=1.0)
        return dict(norms=norms, grads=[t.double() * shrink[:, None] for t in s["grads"]])
    if case["op"] == "rotary":
        # a pair is a complex number, the rotation a product with one of modulus `gain`
        r, x = case["rot"], s["x"].double()
        angle = torch.outer(_positions(s, case).double(), _frequencies(case)) * (-1.0 if case["backward"] else 1.0)
        turn = torch.polar(torch.full_like(angle, RAMP_GAIN if case["scaling"] == "ramp" else GAIN), angle)[:, None, :]
        if case["layout"] == "half":
            y = torch.complex(x[..., : r // 2], x[..., r // 2 : r]) * turn
            head = torch.cat([y.real, y.imag], dim=-1)
        else:
            y = torch.view_as_complex(x[..., :r].reshape(*x.shape[:-1], r // 2, 2).contiguous()) * turn
            head = torch.view_as_real(y).flatten(-2)
        return torch.cat([head, x[..., r:]], dim=-1)
    # block: the definition, its gradients by automatic differentiation
    P, rows, d = case["P"], case["rows"], case["d"]
    leaf = lambda t: t.double().requires_grad_(case["train"])  # noqa: E731
    y, x = leaf(s["y"]), leaf(s["x"])
    params = {k: leaf(v) for k, v in s["params"].items()}
    gate = None if s["gate"] is None else leaf(s["gate"])

    def norm(kind, v, which):
        if kind == "none":
            return v
        if kind == "layer":
            v = (v - v.mean(-1, keepdim=True)) / (v.var(-1, unbiased=False, keepdim=True) + EPS).sqrt()
        else:
            v = v / (v.square().mean(-1, keepdim=True) + EPS).sqrt()
        v = v * params[which + "_gain"].view(P, 1, d)
        return v + params[which + "_bias"].view(P, 1, d) if which + "_bias" in params else v

    act = {"none": lambda g: g, "sigmoid": torch.sigmoid, "silu": lambda g: g * torch.sigmoid(g), "tanh": torch.tanh}[case["act"]]
    u = norm(case["post"], y.view(P, rows, d), "post")
    if case["gate"] == "vector":
        u = u * act(params["gate"]).view(P, 1, d)
    elif case["gate"] == "rows":
        u = u * act(gate).view(P, rows, d)
    out = ALPHA * x.view(P, rows, d) + BETA * u
    z = norm(case["pre"], out, "pre") if case["pre"] != "none" else None
    res = dict(out=out.detach().view(P * rows, d))
    if z is not None:
        res["z"] = z.detach().view(P * rows, d)
    if case["train"]:
        total = (out * s["dout"].double().view(P, rows, d)).sum()
        if z is not None:
            total = total + (z * s["dz"].double().view(P, rows, d)).sum()
        total.backward()
        res.update(dy=y.grad, dx=x.grad, **{"d_" + k: v.grad for k, v in params.items()})
        if gate is not None:
            res["dgate"] = gate.grad
    return res


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "clip":
        n = case["P"] * sum(int(k) for k in case["sizes"].split("-"))
        return {"bytes": 2 * n * BYTES[case["dtype"]] + 8 * case["P"], "flops": 3 * n}
    if case["op"] == "rotary":
        n = case["rows"] * case["heads"] * case["width"]
        pairs = case["rows"] * case["heads"] * case["rot"] // 2
        return {"bytes": 2 * n * BYTES[case["dtype"]] + (0 if case["period"] else 4 * case["rows"]), "flops": 6 * pairs}
    n, a, r = case["P"] * case["rows"] * case["d"], BYTES[case["dtype"]], BYTES[case["res"]]
    gated, normed = case["gate"] == "rows", case["pre"] != "none"
    per = a + 2 * r + (a if normed else 0) + (a if gated else 0)
    flops = 16
    if case["train"]:
        per += a + 2 * r + (a if normed else 0) + (a if gated else 0)
        flops += 34
    params = sum([case["post"] != "none", case["post"] == "layer", normed, case["pre"] == "layer", case["gate"] == "vector"])
    return {"bytes": n * per + params * case["P"] * case["d"] * 4 * (2 if case["train"] else 1), "flops": n * flops}
