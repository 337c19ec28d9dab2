"""Gradient clipping, rotary positions and block norms on the GPU against the float64 oracle.

Tolerances, derived: U = 2^-24 is half a step of float32 and HALF[t] half a step of the output's type, both relative.  Every bound is HALF |value| for the
last rounding plus some U times a magnitude that the arithmetic passed through (a sum of absolute values in place of the sums, so that cancellation is
counted), written at each test."""
import numpy as np
import pytest
import torch

from oracle import operators as oo
from paper_1711_09846_amd import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _cpu(t):
    return t.detach().to("cpu").double().numpy()


def _normal(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def _gen(seed=0):
    return torch.Generator().manual_seed(seed)


def _close(got, want, tol, what):
    err = np.abs(_cpu(got) - want)
    bad = ~(err <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(err / np.maximum(tol, 1e-300))), np.argwhere(bad)[:3].tolist())


# ---- clip ---------------------------------------------------------------------------------------------------------------------------------------------

SIZES = [[1], [7], [8, 1, 9], [100], [2048, 64, 256, 4], [513, 0, 77, 8191], [70001], [3] * 150, [300000, 5, 1000003]]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%dx%d" % (len(s), sum(s)))
@pytest.mark.parametrize("P", [1, 3])
def test_clip(P, sizes, dtype):
    g, dt = _gen(len(sizes) + P), TYPES[dtype]
    # (members 0.. with norms around 0.5, 1, 2; the bound is 1)
    scale = [0.5 * 2 ** i / np.sqrt(max(1, sum(sizes))) for i in range(P)]
    grads = [torch.stack([_normal(g, n, scale=s) for s in scale]).to(dt) for n in sizes]
    want_norm, want = oo.clip([_cpu(t) for t in grads], 1.0)
    bound = torch.ones(P, device="cuda")
    outs = [torch.full_like(t, 7.0) for t in grads]
    norms = binding.GradClip(grads, outs)(bound)
    # the norm is rounded once; the factor once, the product once, then the output's type
    _close(norms, want_norm, 1.01 * U * want_norm, "norm")
    near = np.abs(want_norm - 1.0) < 1e-6      # (either side of the bound is right there)
    for o, w, t in zip(outs, want, grads):
        tol = (HALF[dt] + 2.01 * U) * np.abs(w) + 1e-45
        _close(o, np.where(near[:, None], _cpu(o), w), tol, "clipped")
        for i in np.flatnonzero(want_norm < 1.0 - 1e-6):
            assert torch.equal(o[i], t[i])
    again = binding.GradClip(grads)            # in place, the same bits
    assert torch.equal(again(bound), norms) and all(torch.equal(a, b) for a, b in zip(grads, outs))


def test_clip_tensors_of_one_flat_array_with_rows_at_any_address():
    """Views of [P][stride] rows that start at odd elements, the gaps between them left alone; a column of hyperparameters as bounds."""
    g = _gen(3)
    flat = _normal(g, 5, 1003)
    before = flat.clone()
    views = [flat[:, 1:300], flat[:, 303:304], flat[:, 401:1001]]
    hyper = torch.tensor([[9.0, b, 9.0] for b in (0.0, 1.0, 5.0, 1e9, float("inf"))], device="cuda")
    want_norm, want = oo.clip([_cpu(v) for v in views], _cpu(hyper[:, 1]))
    norms = binding.GradClip(views)(hyper[:, 1])
    _close(norms, want_norm, 1.01 * U * want_norm, "norm")
    for v, w in zip(views, want):
        _close(v, w, 3.01 * U * np.abs(w) + 1e-45, "clipped")
    mask = torch.ones(1003, dtype=torch.bool)
    for lo, hi in ((1, 300), (303, 304), (401, 1001)):
        mask[lo:hi] = False
    assert torch.equal(flat[:, mask.cuda()], before[:, mask.cuda()])
    # into the columns beside them
    wide = _normal(g, 4, 64)
    src, dst = wide[:, :31], wide[:, 32:63]
    keep = src.clone()
    binding.GradClip([src], [dst])(torch.full((1,), 1e-2, device="cuda"))
    _, want = oo.clip([_cpu(keep)], 1e-2)
    assert torch.equal(src, keep)
    _close(dst, want[0], 3.01 * U * np.abs(want[0]), "beside")


def test_clip_values_at_the_ends_of_the_range():
    """Squares that float32 cannot hold, zeros, infinities and NaN; bounds that are NaN or negative (of a zero gradient too)."""
    inf, nan = float("inf"), float("nan")
    rows = torch.tensor([[3e38, -3e38, 1e38, 0], [1e-38, 1e-40, 0, 1e-45], [0, 0, 0, 0], [1, inf, -2, 3], [1, nan, 2, inf], [3, 4, 0, 0], [3, 4, 0, 0], [0, 0, 0, 0]], device="cuda")
    bounds = torch.tensor([1.0, 1e-39, 1.0, 1.0, 1.0, nan, -1.0, -1.0], device="cuda")
    out = torch.empty_like(rows)
    norms = binding.GradClip([rows], [out])(bounds)
    want = np.sqrt((_cpu(rows) ** 2).sum(axis=1))
    assert np.isinf(_cpu(norms)[0]) and _cpu(norms)[3] == inf and np.isnan(_cpu(norms)[4])
    assert np.allclose(_cpu(norms)[[1, 2, 5, 6]], want[[1, 2, 5, 6]], rtol=1e-7, atol=1e-45)
    o = _cpu(out)
    # the factor 1 / 4.4e38 is below the smallest normal float (1.2e-38): it keeps 2^-149 of absolute precision, 2^-150 / 2.3e-39 relative
    assert np.allclose(o[0], _cpu(rows)[0] / want[0], rtol=2.0 ** -150 / 2.2e-39 + 2 * U, atol=0)
    assert o[2].tolist() == [0, 0, 0, 0] and o[5].tolist() == [3, 4, 0, 0] and o[6].tolist() == [0, 0, 0, 0] and o[7].tolist() == [0, 0, 0, 0]
    assert o[3][0] == 0 and o[3][2] == 0 and np.isnan(o[3][1])
    assert o[4][0] == 1 and np.isnan(o[4][1]) and np.isinf(o[4][3])


def test_clip_norms_only_leaves_tensors_alone():
    g = _gen(5)
    t = _normal(g, 2, 5000)
    keep = t.clone()
    norms = torch.zeros(2, device="cuda")
    assert binding.GradClip([t])(norms=norms) is norms
    _close(norms, np.sqrt((_cpu(t) ** 2).sum(axis=1)), 1.01 * U * 100, "norm")
    assert torch.equal(t, keep)


def test_clip_large_members_use_every_offset():
    """A member's tensor of more than 2^31 bytes and a second member behind it."""
    n = (1 << 29) + 11
    t = torch.zeros(2, n, device="cuda")
    t[0, 5], t[0, -1], t[1, 0], t[1, -1] = 3.0, 4.0, 6.0, 8.0
    norms = binding.GradClip([t])(torch.tensor([10.0, 1.0], device="cuda"))
    assert norms.tolist() == [5.0, 10.0]
    assert [t[0, 5].item(), t[0, -1].item()] == [3.0, 4.0] and np.allclose([t[1, 0].item(), t[1, -1].item()], [0.6, 0.8], rtol=3 * U)


def test_clip_refusals():
    a = torch.zeros(2, 8, device="cuda")
    for bad in (lambda: binding.GradClip([]), lambda: binding.GradClip([a, a]), lambda: binding.GradClip([a.half()]), lambda: binding.GradClip([a.cpu()]),
                lambda: binding.GradClip([a, torch.zeros(3, 8, device="cuda")]), lambda: binding.GradClip([a.t()]), lambda: binding.GradClip([a], [a.bfloat16()]),
                lambda: binding.GradClip([a])(torch.ones(3, device="cuda")), lambda: binding.GradClip([a])(torch.ones(2)),
                lambda: binding.GradClip([a])(norms=torch.ones(2, 2, device="cuda")[:, 0])):
        with pytest.raises(ValueError):
            bad()


# ---- rotary -------------------------------------------------------------------------------------------------------------------------------------------

def _rotary_tol(x, pos, freq, layout, gain, dtype):
    """|x a cos - x b sin|: the factors are off by the reduced angle's rounding (2^-27 half turns), sincospi (4 U), the gain (U each) and the position's
    phase (both sides: the frequency and the product, 4 2^-53 of the angle each); the products and their sum by 2 U of |a| + |b|."""
    r = 2 * len(freq)
    phase = 8 * 2.0 ** -53 * np.abs(pos[:, None] * freq)[:, None, :]
    factor = abs(gain) * (np.pi * 2.0 ** -27 + 6 * U + phase)
    first, second = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    mag = np.abs(x[..., first]) + np.abs(x[..., second])
    tol = np.zeros_like(x)
    tol[..., first] = tol[..., second] = mag * (factor + 2 * abs(gain) * U)
    return tol


def _check_rotary(rot, x, pos, settings, dtype, out, backward, what):
    freq_kw = {k: v for k, v in settings.items() if k not in ("layout", "gain")}
    freq = oo.rotary_frequencies(rot, **freq_kw)
    layout, gain = settings.get("layout", "half"), settings.get("gain", 1.0)
    xn, pn = _cpu(x), np.asarray(pos, dtype=np.float64)
    want = oo.rotary(xn, pn, freq, layout, gain, backward)
    tol = _rotary_tol(xn, pn, freq, layout, gain, dtype)
    _close(out, want, tol + np.where(tol > 0, HALF[dtype], 0.0) * (np.abs(want) + tol), what)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,width,rot", [(1, 1, 2, 2), (1, 16, 64, 64), (3, 5, 84, 42), (17, 2, 128, 64), (130, 3, 20, 18), (5, 1, 300, 256), (2, 4, 513, 512), (33, 40, 16, 8),
                                                  (1000, 7, 10, 6)])
def test_rotary(dtype, layout, rows, heads, width, rot):
    g, dt = _gen(rows + width), TYPES[dtype]
    x = _normal(g, rows, heads, width, dtype=dt)
    pos = torch.randint(0, 5000, (rows,), generator=g)
    r = binding.Rotary(rot, layout=layout)
    keep = x.clone()
    for backward in (False, True):
        out = r(x, torch.full_like(x, 9.0), positions=pos.int().cuda(), backward=backward)
        _check_rotary(rot, x, pos, dict(layout=layout), dt, out, backward, "apart")
    assert torch.equal(x, keep)
    assert r(x, positions=pos.cuda(), backward=True) is x and torch.equal(x, out)      # in place, 64-bit positions: the same bits


@pytest.mark.parametrize("settings", [dict(scaling="linear", factor=8.0), dict(scaling="base", factor=8.0), dict(scaling="ramp", factor=8.0, trained=4096.0, gain=1.2),
                                      dict(base=500000.0, gain=-0.5)], ids=["linear", "base", "ramp", "gain"])
def test_rotary_far_positions_and_scaling(settings):
    g = _gen(7)
    x = _normal(g, 64, 2, 64)
    pos = torch.randint(0, 1 << 20, (64,), generator=g)
    pos[:6] = torch.tensor([0, 1, (1 << 31) - 1, 1 << 30, (1 << 20) - 1, -5])
    out = binding.Rotary(64, **settings)(x, torch.empty_like(x), positions=pos.int().cuda())
    _check_rotary(64, x, pos, settings, torch.float32, out, False, str(settings))


def test_rotary_positions_without_a_tensor():
    g = _gen(8)
    x = _normal(g, 50, 3, 32)
    r = binding.Rotary(32)
    for start, period, pos in ((0, 0, np.arange(50)), (1000, 0, 1000 + np.arange(50)), (0, 16, np.arange(50) % 16), (7, 1, np.full(50, 7)), (3, 50, 3 + np.arange(50))):
        _check_rotary(32, x, pos, {}, torch.float32, r(x, torch.empty_like(x), start=start, period=period), False, (start, period))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rotary_of_query_and_key_heads_inside_a_joint_projection(dtype):
    """8 query heads and 2 key heads of rows that also hold values, at odd addresses and pitches; what is not turned stays as it was."""
    g, dt = _gen(9), TYPES[dtype]
    joint = _normal(g, 40, 1 + 12 * 24 + 2, dtype=dt)
    keep = joint.clone()
    part = lambda t, h0, n: t[:, 1 + h0 * 24:1 + (h0 + n) * 24].unflatten(1, (n, 24))  # noqa: E731
    r = binding.Rotary(16, layout="interleaved")
    r([part(joint, 0, 8), part(joint, 8, 2)], period=8)
    for h0, n in ((0, 8), (8, 2)):
        _check_rotary(16, part(keep, h0, n), np.arange(40) % 8, dict(layout="interleaved"), dt, part(joint, h0, n), False, "group")
    mask = torch.zeros(joint.shape[1], dtype=torch.bool)
    mask[0], mask[1 + 10 * 24:] = True, True
    assert torch.equal(joint[:, mask.cuda()], keep[:, mask.cuda()])
    # heads outermost: [heads, rows, width] memory
    x = _normal(g, 3, 40, 24, dtype=dt)
    out = r(x.transpose(0, 1), torch.empty_like(x).transpose(0, 1), period=8)
    assert torch.equal(out, r(x.transpose(0, 1).contiguous(), torch.empty(40, 3, 24, dtype=dt, device="cuda"), period=8))


def test_rotary_of_many_rows_and_far_offsets():
    """More rows than a grid of one workgroup a row holds, and rows 2^31 bytes from the first."""
    n = 20_000_003
    x = torch.ones(n, 1, 2, device="cuda")
    r = binding.Rotary(2)
    out = r(x, torch.empty_like(x), period=1000)
    at = torch.tensor([0, 999, 1000, 16_777_215, 16_777_217, n - 1], device="cuda")
    _check_rotary(2, x[at], _cpu(at) % 1000, {}, torch.float32, out[at], False, "rows")
    big = torch.zeros(3, 1 << 30, dtype=torch.bfloat16, device="cuda")
    view = big[:, -64:].unflatten(1, (1, 64))
    view.copy_(torch.ones_like(view))
    got = r2 = binding.Rotary(64)(view, start=5)
    _check_rotary(64, torch.ones(3, 1, 64), [5, 6, 7], {}, torch.bfloat16, got, False, "offsets")
    assert r2 is view and not big[:, :-64].any()


def test_rotary_infinities_stay_in_their_pairs():
    x = torch.ones(2, 2, 8, device="cuda")
    x[0, 0, 1], x[1, 1, 7] = float("inf"), float("nan")
    out = _cpu(binding.Rotary(4)(x, torch.empty_like(x), start=3))
    finite = np.ones((2, 2, 8), dtype=bool)
    finite[0, 0, [1, 3]], finite[1, 1, 7] = False, False
    assert np.array_equal(np.isfinite(out), finite)


def test_rotary_refusals():
    x = torch.zeros(4, 2, 8, device="cuda")
    r = binding.Rotary(8)
    with pytest.raises(ValueError):
        binding.Rotary(8, layout="both")
    for bad in (lambda: r(x[0]), lambda: r(x.half()), lambda: r(x, x.bfloat16()), lambda: r(x, positions=torch.zeros(3, dtype=torch.int32, device="cuda")),
                lambda: r(x, positions=torch.zeros(4, device="cuda")), lambda: r(x.transpose(1, 2)), lambda: r([x], []), lambda: r(x.cpu())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: binding.Rotary(7), lambda: r(x[..., :6]), lambda: r(x[:3], x[1:]), lambda: r(x.expand(4, 2, 8)[:1].expand(4, 2, 8))):
        with pytest.raises(binding.PbtError):
            bad()
    assert r(x[:0]).shape[0] == 0


# ---- block norms --------------------------------------------------------------------------------------------------------------------------------------

def _case(P, rows, d, post, pre, gate, act, dtype, res, seed=0):
    g, dt, rt = _gen(seed + d + rows), TYPES[dtype], TYPES[res]
    n = P * rows
    params = {}
    if post != "none":
        params.update(post_gain=1 + _normal(g, P, d, scale=0.2), post_bias=_normal(g, P, d, scale=0.2))
    if pre != "none":
        params.update(pre_gain=1 + _normal(g, P, d, scale=0.2), pre_bias=_normal(g, P, d, scale=0.2))
    if gate == "vector":
        params["gate"] = _normal(g, P, d)
    return dict(y=0.3 + _normal(g, n, d, dtype=dt), x=_normal(g, n, d, scale=2.0, dtype=rt) - 0.5, gate=_normal(g, n, d, scale=1.5, dtype=dt) if gate == "rows" else None,
                dout=_normal(g, n, d, dtype=rt), dz=_normal(g, n, d, dtype=dt) if pre != "none" else None, params=params)


def _magnitudes(spec, y, x, p, gate, dout, dz):
    """Sums of absolute values that the float32 arithmetic of one member passes through: of u, out, z, and t, dgate, dy, and per column of the sums.

    A row's mean is off by U times the mean absolute value (times the length of a chain of sums), 1 / spread relatively by as much as the squares' sum."""
    row = lambda v: v.mean(axis=-1, keepdims=True)  # noqa: E731
    o64, z64, (_, u, f, df, c1, c2) = spec.forward(y, x, p, gate)
    f, df = np.abs(f), np.abs(df)
    m = {}
    if spec.post != "none":
        yh, r1 = np.abs(c1[0]), c1[1]
        m_yh = yh + r1 * row(np.abs(y)) * (1 + yh) if spec.post == "layer" else yh       # what 64 U of error in yh is relative to
        m_u = np.abs(p["post_gain"]) * m_yh + np.abs(p["post_bias"])
    else:
        m_yh = m_u = np.abs(u)
    m["out"] = abs(spec.alpha) * np.abs(x) + abs(spec.beta) * f * m_u
    if spec.pre != "none":
        xh, r2 = np.abs(c2[0]), c2[1]
        spread = r2 * np.sqrt(row(m["out"] ** 2))      # error of out in units of the spread
        m_xh = xh * (1 + spread) + r2 * (m["out"] + row(m["out"]))
        m["z"] = np.abs(p["pre_gain"]) * m_xh + np.abs(p["pre_bias"])
    if dout is None and dz is None:
        return m
    t = np.zeros_like(o64) if dout is None else np.abs(dout)
    if spec.pre != "none" and dz is not None:
        w = np.abs(dz * p["pre_gain"])
        s = row(w * m_xh)
        t = t + r2 * (1 + spread) * (w + row(w) + m_xh * s)
        m["pre_gain"], m["pre_bias"] = (np.abs(dz) * m_xh).sum(0), np.abs(dz).sum(0)
    m["dx"] = abs(spec.alpha) * t
    v = abs(spec.beta) * f * t
    m["dgate"] = abs(spec.beta) * df * m_u * t
    m["gate"] = m["dgate"].sum(0)
    if spec.post != "none":
        w = v * np.abs(p["post_gain"])
        m["dy"] = r1 * (1 + (r1 * row(np.abs(y)) if spec.post == "layer" else 0)) * (w + row(w) + m_yh * row(w * m_yh))
        m["post_gain"], m["post_bias"] = (v * m_yh).sum(0), v.sum(0)
    else:
        m["dy"] = v
    return m


# a row's sum is a chain of at most 16 additions in a lane and 9 across lanes and wavefronts, twice (mean, squares), then some ten operations and two
# function calls of a few U: 64 U of the magnitudes; a column's sum is a chain of at most `rows` additions on top
CHAIN = 64


def _check_block(c, P, rows, d, post, pre, gate, act, dtype, res, alpha=0.9, beta=0.7, have=("dout", "dz")):
    dt, rt = TYPES[dtype], TYPES[res]
    op = binding.BlockNorm(d, members=P, post=post, pre=pre, gate=gate, act=act, alpha=alpha, beta=beta)
    spec = oo.BlockNorm(post, pre, gate, act, alpha=alpha, beta=beta)
    keep = {k: v.clone() for k, v in c.items() if isinstance(v, torch.Tensor)}
    out, z, stats = op.forward(c["y"], c["x"], c["params"], gate=c["gate"])
    dout, dz = (c["dout"] if "dout" in have else None), (c["dz"] if "dz" in have else None)
    dy, dx, dgate, grads = op.backward(c["y"], c["x"], c["params"], stats, dout, dz, gate=c["gate"])
    assert all(torch.equal(c[k], v) for k, v in keep.items())
    assert set(grads) == set(c["params"])
    for i in range(P):
        part = lambda t: None if t is None else _cpu(t[i * rows:(i + 1) * rows])  # noqa: E731
        p = {k: _cpu(v[i]) for k, v in c["params"].items()}
        w_out, w_z, cache = spec.forward(part(c["y"]), part(c["x"]), p, part(c["gate"]))
        w_dy, w_dx, w_dgate, w_grads = spec.backward(cache, part(dout), part(dz))
        m = _magnitudes(spec, part(c["y"]), part(c["x"]), p, part(c["gate"]), part(dout), part(dz))

        def check(got, want, name, t, chain=CHAIN):
            _close(got[i * rows:(i + 1) * rows], want, HALF[t] * np.abs(want) + 1.01 * chain * U * m[name], (name, i))

        check(out, w_out, "out", rt)
        if z is not None:
            check(z, w_z, "z", dt)
        check(dy, w_dy, "dy", dt)
        check(dx, w_dx, "dx", rt)
        if dgate is not None:
            check(dgate, w_dgate, "dgate", dt)
        for k, v in grads.items():
            if k.startswith("pre") and dz is None:
                assert not v.any()
                continue
            _close(v[i], w_grads[k], (CHAIN + rows) * U * m[k], (k, i))


SHAPES = [(1, 1, 1), (1, 1, 8), (2, 3, 5), (3, 70, 7), (2, 33, 64), (1, 65, 61), (2, 40, 200), (1, 9, 256), (1, 5, 128), (3, 7, 130), (1, 33, 512), (2, 9, 513), (1, 4, 1024), (1, 3, 1500), (2, 5, 1025), (1, 4, 4609), (1, 2, 2048), (2, 2, 4095), (1, 3, 5001), (1, 2, 8192), (2, 700, 24)]


@pytest.mark.parametrize("P,rows,d", SHAPES)
@pytest.mark.parametrize("dtype,res", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16")])
def test_block_norm_shapes_and_types(P, rows, d, dtype, res):
    kw = dict(post="rms", pre="layer", gate="rows", act="sigmoid", dtype=dtype, res=res)
    _check_block(_case(P, rows, d, **kw), P, rows, d, **kw)


@pytest.mark.parametrize("post,pre", [("layer", "layer"), ("rms", "rms"), ("layer", "rms"), ("none", "layer"), ("none", "rms"), ("layer", "none"), ("rms", "none")])
@pytest.mark.parametrize("gate,act", [("none", "none"), ("vector", "none"), ("vector", "silu"), ("rows", "none"), ("rows", "silu"), ("rows", "tanh"), ("vector", "sigmoid")])
def test_block_norm_kinds(post, pre, gate, act):
    for P, rows, d in ((2, 13, 72), (1, 5, 1031)):
        kw = dict(post=post, pre=pre, gate=gate, act=act, dtype="bf16", res="fp32")
        _check_block(_case(P, rows, d, **kw), P, rows, d, **kw)


@pytest.mark.parametrize("have", [("dout",), ("dz",)])
def test_block_norm_backward_of_one_output(have):
    kw = dict(post="layer", pre="rms", gate="vector", act="tanh", dtype="bf16", res="bf16")
    _check_block(_case(2, 6, 200, **kw), 2, 6, 200, have=have, **kw)


def test_block_norm_without_parameters_and_without_statistics():
    c = _case(1, 9, 100, "layer", "rms", "none", "none", "fp32", "fp32")
    c["params"] = {}
    op = binding.BlockNorm(100, post="layer", pre="rms")
    out, z, stats = op.forward(c["y"], c["x"], stats=False)
    assert stats is None
    ones = dict(post_gain=torch.ones(100, device="cuda"), post_bias=torch.zeros(100, device="cuda"), pre_gain=torch.ones(100, device="cuda"))
    out2, z2, stats = op.forward(c["y"], c["x"], ones)
    assert torch.equal(out, out2) and torch.equal(z, z2)
    a = op.backward(c["y"], c["x"], {}, stats, c["dout"], c["dz"])
    b = op.backward(c["y"], c["x"], ones, stats, c["dout"], c["dz"])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and a[3] == {} and set(b[3]) == set(ones)


def test_block_norm_in_place_strided_rows_and_parameters_of_a_flat_store():
    """out over x, z over y, dx over dout, dy over dz, rows at odd pitches and addresses, parameters inside [P][stride] rows, and the memory between."""
    P, rows, d = 2, 11, 70
    c = _case(P, rows, d, "rms", "layer", "vector", "none", "bf16", "fp32")
    op = binding.BlockNorm(d, members=P, post="rms", pre="layer", gate="vector", alpha=0.9, beta=0.7)
    out, z, stats = op.forward(c["y"], c["x"], c["params"])
    dy, dx, _, grads = op.backward(c["y"], c["x"], c["params"], stats, c["dout"], c["dz"])

    def strided(t, pitch=77, first=3):
        big = torch.full((t.shape[0], pitch), 5.0, dtype=t.dtype, device="cuda")
        big[:, first:first + d] = t
        return big, big[:, first:first + d]

    store, gstore = torch.full((P, 513), 3.0, device="cuda"), torch.full((P, 513), 4.0, device="cuda")
    params, g2 = {}, {}
    for k, (name, v) in enumerate(c["params"].items()):
        store[:, 1 + 90 * k:1 + 90 * k + d] = v
        params[name], g2[name] = store[:, 1 + 90 * k:1 + 90 * k + d], gstore[:, 1 + 90 * k:1 + 90 * k + d]
    ybig, y = strided(c["y"])
    xbig, x = strided(c["x"], 75, 1)
    op.forward(y, x, params, out=x, z=y)
    assert torch.equal(x, out) and torch.equal(y, z)
    assert (ybig[:, :3] == 5).all() and (ybig[:, 73:] == 5).all() and (xbig[:, :1] == 5).all() and (xbig[:, 71:] == 5).all()
    dzbig, dz = strided(c["dz"])
    dobig, do = strided(c["dout"])
    op.backward(strided(c["y"])[1], strided(c["x"])[1], params, stats, do, dz, dy=dz, dx=do, grads=g2)
    assert torch.equal(dz, dy) and torch.equal(do, dx) and all(torch.equal(g2[k], grads[k]) for k in grads)
    mask = torch.ones(513, dtype=torch.bool)
    for k in range(len(params)):
        mask[1 + 90 * k:1 + 90 * k + d] = False
    assert (gstore[:, mask.cuda()] == 4).all() and (dzbig[:, 73:] == 5).all() and (dobig[:, :3] == 5).all()


def test_block_norm_rows_that_are_constant_or_not_finite():
    """A constant row has spread sqrt(eps); a row with an infinity or NaN spoils itself and the columns' sums only."""
    d = 40
    y = torch.randn(4, d, generator=_gen(1)).cuda()
    x = torch.randn(4, d, generator=_gen(2)).cuda()
    y[0], x[0] = 3.0, 1.0
    y[2, 5] = float("inf")
    y[3, 7] = float("nan")
    op, spec = binding.BlockNorm(d), oo.BlockNorm()
    out, z, stats = op.forward(y, x)
    want_out, want_z, _ = spec.forward(_cpu(y)[:2], _cpu(x)[:2], {})
    # (the constant row: u is exactly 0, out exactly 1, z exactly 0)
    assert (out[0] == 1).all() and (z[0] == 0).all()
    assert np.allclose(_cpu(out)[1], want_out[1], atol=1e-5) and np.allclose(_cpu(z)[1], want_z[1], atol=1e-5)
    assert not torch.isfinite(z[2:]).any() and torch.isfinite(z[:2]).all()
    dy, dx, _, _ = op.backward(y, x, {}, stats, torch.ones_like(x), torch.ones_like(y))
    assert torch.isfinite(dy[:2]).all() and torch.isfinite(dx[:2]).all()


def test_block_norm_gradients_against_differences_of_the_kernel():
    """The forward kernel in fp32 along a direction, central difference with h = 2^-6: truncation h^2 / 6 times a third derivative of a few times the sum of
    absolute products, rounding 64 U / h of it."""
    P, rows, d = 1, 6, 48
    kw = dict(post="layer", pre="rms", gate="rows", act="silu", dtype="fp32", res="fp32")
    c = _case(P, rows, d, **kw)
    op = binding.BlockNorm(d, post="layer", pre="rms", gate="rows", act="silu")
    _, _, stats = op.forward(c["y"], c["x"], c["params"], gate=c["gate"])
    dy, dx, dgate, grads = op.backward(c["y"], c["x"], c["params"], stats, c["dout"], c["dz"], gate=c["gate"])
    h = 2.0 ** -6
    value = lambda y, x, gate, p: sum((_cpu(a) * _cpu(b)).sum() for a, b in zip(op.forward(y, x, p, gate=gate)[:2], (c["dout"], c["dz"])))  # noqa: E731
    total = float(c["dout"].abs().sum() + c["dz"].abs().sum())
    for name, grad in [("y", dy), ("x", dx), ("gate", dgate)] + [(k, v) for k, v in grads.items()]:
        base = c["params"][name] if name in c["params"] else c[name]
        v = torch.randn(base.shape, generator=_gen(4)).cuda()
        v /= v.norm() / np.sqrt(rows)

        def at(s):
            moved = dict(y=c["y"], x=c["x"], gate=c["gate"])
            p = dict(c["params"])
            (p if name in p else moved)[name] = base + s * h * v
            return value(moved["y"], moved["x"], moved["gate"], p)

        slope = (at(1) - at(-1)) / (2 * h)
        assert abs(slope - (_cpu(grad) * _cpu(v)).sum()) <= total * (h * h + 64 * U / h), name


def test_block_norm_refusals():
    y = torch.zeros(4, 16, device="cuda")
    op = binding.BlockNorm(16, members=2, gate="rows")
    for bad in (lambda: binding.BlockNorm(16, post="group"), lambda: op.forward(y[:3], y[:3], gate=y[:3]), lambda: op.forward(y, y[:2], gate=y), lambda: op.forward(y.half(), y, gate=y),
                lambda: op.forward(y, y, dict(scale=y), gate=y), lambda: op.forward(y, y, dict(pre_gain=torch.zeros(3, 16, device="cuda")), gate=y),
                lambda: op.forward(y.t().contiguous().t(), y, gate=y), lambda: op.forward(y, y, gate=y.bfloat16())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: binding.BlockNorm(16, post="none", pre="none"), lambda: binding.BlockNorm(9000), lambda: op.forward(y, y), lambda: op.forward(y, y + 1, gate=y, out=y)):
        with pytest.raises(binding.PbtError):
            bad()
    empty = op.forward(y[:0], y[:0], gate=y[:0])
    assert empty[0].shape == (0, 16)
    params = dict(pre_gain=torch.ones(2, 16, device="cuda"))
    grads = op.backward(y[:0], y[:0], params, empty[2], y[:0], y[:0], gate=y[:0])[3]
    assert not grads["pre_gain"].any()


# ---- together, on streams and in graphs -----------------------------------------------------------------------------------------------------------------

def _layer(P=2, rows=48, heads=2, width=32, seed=11):
    """Projections turned by their positions, a block norm forward and backward, the rotation's transpose and the clipped gradients."""
    d = heads * width
    g = _gen(seed)
    c = _case(P, rows, d, "rms", "layer", "vector", "none", "bf16", "bf16", seed)
    qkv = _normal(g, P * rows, 3 * d, dtype=torch.bfloat16)
    dqkv = _normal(g, P * rows, 3 * d, dtype=torch.bfloat16)
    grads = {k: torch.empty(P, d, device="cuda") for k in c["params"]}
    rot, op = binding.Rotary(width), binding.BlockNorm(d, members=P, post="rms", pre="layer", gate="vector")
    clip = binding.GradClip(list(grads.values()))
    bound = torch.full((P,), 0.5, device="cuda")
    heads_of = lambda t: t[:, :2 * d].unflatten(1, (2 * heads, width))  # noqa: E731

    def run():
        turned = rot(heads_of(qkv), torch.empty(P * rows, 2 * heads, width, dtype=torch.bfloat16, device="cuda"), period=16)
        out, z, stats = op.forward(c["y"], c["x"], c["params"])
        dy, dx, _, _ = op.backward(c["y"], c["x"], c["params"], stats, c["dout"], c["dz"], grads=grads)
        back = rot(heads_of(dqkv), torch.empty(P * rows, 2 * heads, width, dtype=torch.bfloat16, device="cuda"), period=16, backward=True)
        norms = clip(bound)
        return [turned, out, z, dy, dx, back, norms] + list(grads.values())

    return run, (c, qkv, dqkv)


def test_operators_together():
    run, _ = _layer()
    first = [t.clone() for t in run()]
    again = run()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    norms, grads = first[6], first[7:]
    after = torch.stack([g.double().square().sum(1) for g in grads]).sum(0).sqrt()
    assert (norms > 0.5).all() and np.allclose(_cpu(after), 0.5, rtol=4 * U)


def test_operators_on_another_stream_and_in_graphs():
    """Two captured graphs of the same calls, replayed in turn with eager work and new inputs between, equal the eager results every time."""
    run, state = _layer()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = run()
        graphs.append((g, outs))
    c, qkv, dqkv = state
    for k in range(4):
        for t in (c["y"], c["x"], c["dz"], c["dout"], qkv, dqkv):
            t.copy_(torch.randn(t.shape, generator=_gen(20 + k)))
        eager = [t.clone() for t in run()]
        torch.cuda.synchronize()
        g, outs = graphs[k % 2]
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, outs)), k


@pytest.mark.parametrize("names", [("post_gain", "pre_gain"), ("post_gain",), ("pre_bias", "gate"), ()])
def test_block_norm_some_parameters_of_wide_rows(names):
    """Which parameters' gradients are asked for does not change the others, at a width whose backward kernel depends on it."""
    P, rows, d = 2, 5, 6200
    c = _case(P, rows, d, "layer", "layer", "vector", "none", "bf16", "fp32")
    op = binding.BlockNorm(d, members=P, post="layer", pre="layer", gate="vector")
    _, _, stats = op.forward(c["y"], c["x"], c["params"])
    dy, dx, _, grads = op.backward(c["y"], c["x"], c["params"], stats, c["dout"], c["dz"])
    some = {k: torch.full_like(grads[k], 9.0) for k in names}
    dy2, dx2, _, _ = op.backward(c["y"], c["x"], c["params"], stats, c["dout"], c["dz"], grads=some)
    assert torch.equal(dy, dy2) and torch.equal(dx, dx2) and all(torch.equal(some[k], grads[k]) for k in names)


@pytest.mark.parametrize("d", [5, 61, 513, 519, 1027, 4099, 5001])
@pytest.mark.parametrize("post,pre", [("none", "rms"), ("layer", "none"), ("rms", "layer")])
def test_block_norm_over_its_inputs_at_widths_that_end_anywhere(d, post, pre):
    """out over x, z over y, dx over dout, dy over dz, where the lane at a row's end shares its eight elements with its neighbours: the same bits as apart."""
    rows = 37
    c = _case(1, rows, d, post, pre, "rows", "sigmoid", "bf16", "bf16")
    op = binding.BlockNorm(d, post=post, pre=pre, gate="rows", act="sigmoid")
    out, z, stats = op.forward(c["y"], c["x"], c["params"], gate=c["gate"])
    dy, dx, dgate, grads = op.backward(c["y"], c["x"], c["params"], stats, c["dout"], c["dz"], gate=c["gate"])
    y, x = c["y"].clone(), c["x"].clone()
    _, _, stats2 = op.forward(y, x, c["params"], gate=c["gate"], out=x, z=y)
    assert torch.equal(x, out) and torch.equal(stats, stats2) and (z is None or torch.equal(y, z))
    dout, dz = c["dout"].clone(), None if c["dz"] is None else c["dz"].clone()
    dy2, _, dgate2, grads2 = op.backward(c["y"], c["x"], c["params"], stats, dout, dz, gate=c["gate"], dy=dz, dx=dout)
    assert torch.equal(dout, dx) and torch.equal(dy2, dy) and torch.equal(dgate, dgate2) and all(torch.equal(grads[k], grads2[k]) for k in grads)


def test_rotary_of_one_groups_heads_twice_is_refused():
    x = torch.zeros(4, 2, 8, device="cuda")
    r = binding.Rotary(8)
    for src, dst in (([x, x], None), ([x, x[:, :1]], None), ([x, x.clone()], [torch.empty_like(x), x])):
        with pytest.raises(binding.PbtError):
            r(src, dst)


def test_block_norm_rows_far_apart():
    """Rows 2^31 bytes from one another, forward and backward; nothing between them is written."""
    P, rows, d = 1, 3, 72
    kw = dict(post="rms", pre="layer", gate="rows", act="sigmoid")
    c = _case(P, rows, d, dtype="bf16", res="bf16", **kw)
    op = binding.BlockNorm(d, **kw)
    out, z, stats = op.forward(c["y"], c["x"], c["params"], gate=c["gate"])
    dy, dx, dgate, _ = op.backward(c["y"], c["x"], c["params"], stats, c["dout"], c["dz"], gate=c["gate"])
    big = torch.zeros(rows, 1 << 30, dtype=torch.bfloat16, device="cuda")
    at = iter(range(0, 9 * 128, 128))

    def far(t=None):
        k = (1 << 30) - 2000 + next(at)
        v = big[:, k:k + d]
        if t is not None:
            v.copy_(t)
        return v

    y, x, gate = far(c["y"]), far(c["x"]), far(c["gate"])
    out2, z2, stats2 = op.forward(y, x, c["params"], gate=gate, out=far(), z=far())
    dout, dz = far(c["dout"]), far(c["dz"])
    dy2, dx2, dgate2, _ = op.backward(y, x, c["params"], stats2, dout, dz, gate=gate, dy=dz, dx=dout, dgate=far())
    for a, b in ((out, out2), (z, z2), (stats, stats2), (dy, dy2), (dx, dx2), (dgate, dgate2)):
        assert torch.equal(a, b)
    assert not big[:, :(1 << 30) - 2000].any() and not big[:, -600:].any()


def test_block_norm_gate_matrix_needs_its_kind():
    y = torch.zeros(2, 16, device="cuda")
    op = binding.BlockNorm(16)
    with pytest.raises(ValueError):
        op.forward(y, y, gate=y)
    stats = op.forward(y, y)[2]
    for kw in (dict(gate=y), dict(dgate=y)):
        with pytest.raises(ValueError):
            op.backward(y, y, {}, stats, y, y, **kw)
