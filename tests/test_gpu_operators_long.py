"""The operators where their kernels go round their loops: several rows a team, several rows of angles a workgroup, several units a thread, several tables, results
past the caches (operator_cases.py), against the float64 oracle.

Tolerances as in test_gpu_operators.py: half a step of the output's type plus a counted number of half steps of float32 times what the arithmetic passes
through."""
import numpy as np
import pytest
import torch

from oracle import operators as oo
from paper_1711_09846_amd import binding
from tests import native_operators as rules, operator_cases
from tests.test_gpu_operators import CHAIN, HALF, TYPES, U, _case, _close, _cpu, _gen, _magnitudes, _normal

pytestmark = pytest.mark.gpu


def _name(c):
    return "-".join(str(v) for v in c.values()).replace(" ", "")


# ---- block norms ----

def _block_case(c):
    names = operator_cases.block_params(c)
    t = _case(c["P"], c["rows"], c["d"], c["post"], c["pre"], c["gate"], c["act"], c["dtype"], c["res"])
    t["params"] = {k: v for k, v in t["params"].items() if k in names}
    op = binding.BlockNorm(c["d"], members=c["P"], post=c["post"], pre=c["pre"], gate=c["gate"], act=c["act"], alpha=0.9, beta=0.7)
    return t, op


@pytest.mark.parametrize("c", operator_cases.BLOCK, ids=_name)
def test_block_norm_of_several_rows_a_team(c):
    """Rows as in test_gpu_operators.py (CHAIN: what their sums count).  A column's sum: a team adds its rows of a slab in turn, the teams of a workgroup are joined in
    at most 3 + 3 additions, a quarter of the slabs in turn and the quarters in three: that many half steps on top of CHAIN."""
    P, rows, d = c["P"], c["rows"], c["d"]
    t, op = _block_case(c)
    spec = oo.BlockNorm(c["post"], c["pre"], c["gate"], c["act"], alpha=0.9, beta=0.7)
    cut = rules.block(P, rows, d, c["post"], c["pre"], c["gate"], c["dtype"], c["res"], len(t["params"]))
    chain = CHAIN + -(-cut.backward // cut.team_rows) + 6 + -(--(-rows // cut.backward) // 4) + 3
    out, z, stats = op.forward(t["y"], t["x"], t["params"], gate=t["gate"])
    dy, dx, dgate, grads = op.backward(t["y"], t["x"], t["params"], stats, t["dout"], t["dz"], gate=t["gate"])
    dt, rt = TYPES[c["dtype"]], TYPES[c["res"]]
    for i in range(P):
        part = lambda v: None if v is None else _cpu(v[i * rows:(i + 1) * rows])  # noqa: E731
        p = {k: _cpu(v[i]) for k, v in t["params"].items()}
        full = dict(post_gain=np.ones(d), post_bias=np.zeros(d), pre_gain=np.ones(d), pre_bias=np.zeros(d))
        full.update(p)
        y, x, gate, dout, dz = (part(t[k]) for k in ("y", "x", "gate", "dout", "dz"))
        w_out, w_z, cache = spec.forward(y, x, p, gate)
        w_dy, w_dx, w_dgate, w_grads = spec.backward(cache, dout, dz)
        m = _magnitudes(spec, y, x, full, gate, dout, dz)
        for got, want, name, ty in ((out, w_out, "out", rt), (z, w_z, "z", dt), (dy, w_dy, "dy", dt), (dx, w_dx, "dx", rt), (dgate, w_dgate, "dgate", dt)):
            if got is not None:
                _close(got[i * rows:(i + 1) * rows], want, HALF[ty] * np.abs(want) + 1.01 * CHAIN * U * m[name], (name, i))
        assert set(grads) == set(t["params"])
        for k, v in grads.items():
            _close(v[i], w_grads[k], chain * U * m[k], (k, i))


@pytest.mark.parametrize("c", operator_cases.BLOCK, ids=_name)
def test_block_norm_of_several_rows_a_team_over_its_inputs(c):
    """out over x, z over y, dx over dout, dy over dz while the next rows are on their way: the same bits as apart."""
    t, op = _block_case(c)
    out, z, stats = op.forward(t["y"], t["x"], t["params"], gate=t["gate"])
    dy, dx, dgate, grads = op.backward(t["y"], t["x"], t["params"], stats, t["dout"], t["dz"], gate=t["gate"])
    y, x = t["y"].clone(), t["x"].clone()
    _, _, stats2 = op.forward(y, x, t["params"], gate=t["gate"], out=x, z=y)
    assert torch.equal(x, out) and torch.equal(stats, stats2) and (z is None or torch.equal(y, z))
    dout, dz = t["dout"].clone(), None if t["dz"] is None else t["dz"].clone()
    dy2, _, dgate2, grads2 = op.backward(t["y"], t["x"], t["params"], stats, dout, dz, gate=t["gate"], dy=dz, dx=dout)
    assert torch.equal(dout, dx) and torch.equal(dy2, dy) and (dgate is None or torch.equal(dgate, dgate2)) and all(torch.equal(grads[k], grads2[k]) for k in grads)


# ---- rotary ----

def _turned(x, pos, rot, layout, backward=False, base=10000.0):
    """(the oracle's values, their tolerance).  Angle in quarter turns: rounded to float, times a rounded pi / 2, rounded: 3 U of at most pi / 4, which moves sine
    and cosine by at most 1.7 U.  Their series by fused steps: at most 1.2 U, with 2e-9 for what it leaves out.  Gain and its product 2 U, phase of far positions
    8 2^-53 of the angle.  Then a product of each and their sum: 2 U of |a| + |b|.  In all 7 U and the phase, of |a| + |b|."""
    freq = oo.rotary_frequencies(rot, base=base)
    xn, pn = _cpu(x), np.asarray(pos, dtype=np.float64)
    want = oo.rotary(xn, pn, freq, layout, 1.0, backward)
    first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    tol = np.zeros_like(xn)
    tol[..., first] = tol[..., second] = (np.abs(xn[..., first]) + np.abs(xn[..., second])) * (7 * U + 8 * 2.0 ** -53 * np.abs(pn[:, None] * freq)[:, None, :])
    return want, tol + np.where(tol > 0, HALF[x.dtype], 0.0) * (np.abs(want) + tol)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("c", operator_cases.ROTARY, ids=_name)
def test_rotary_of_several_rows_a_workgroup(c, layout, dtype):
    g, dt = _gen(c["rows"] + c["width"]), TYPES[dtype]
    joint = _normal(g, c["rows"], sum(c["heads"]) + 1, c["width"], dtype=dt)
    keep = joint.clone()
    pos = torch.randint(0, 5000, (c["rows"],), generator=g, dtype=torch.int32)
    srcs = list(torch.split(joint[:, :-1], c["heads"], dim=1))
    outs = [torch.full((c["rows"], h, c["width"]), 9.0, dtype=dt, device="cuda") for h in c["heads"]] if c["apart"] else srcs
    binding.Rotary(c["rot"], layout=layout)(srcs, outs, positions=pos.cuda())
    assert torch.equal(joint[:, -1], keep[:, -1]) and (not c["apart"] or torch.equal(joint, keep))
    at = 0
    for out, h in zip(outs, c["heads"]):
        heads = range(h) if h < 20 else [0, 1, 255, 256, 408, 409, 511, 512, h - 1]       # (of many heads some, around the workgroups' borders)
        for k in heads:
            want, tol = _turned(keep[:, at + k:at + k + 1], pos, c["rot"], layout)
            _close(out[:, k:k + 1], want, tol, ("head", k))
        at += h


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_past_the_caches_at_odd_addresses(layout):
    """A call of more than 256 MB from odd elements to odd elements: the bits of the same rows turned in small calls, which the oracle looks at."""
    rows, heads, w, rot = 140001, 16, 64, 42
    x = torch.randn(rows * heads * w + 1, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()[1:].view(rows, heads, w)
    out = torch.empty(rows * heads * w + 3, dtype=torch.bfloat16, device="cuda")[3:].view(rows, heads, w)
    r = binding.Rotary(rot, layout=layout)
    r(x, out, start=11)
    for lo in range(0, rows, 30000):
        part = x[lo:lo + 30000].clone()
        assert torch.equal(out[lo:lo + 30000], r(part, torch.empty_like(part), start=11 + lo)), lo
    at = torch.tensor([0, 1, 77777, rows - 1], device="cuda")
    want, tol = _turned(x[at], 11 + _cpu(at), rot, layout)
    _close(out[at], want, tol, "rows")


def test_rotary_of_more_rows_than_two_million_workgroups_hold():
    """Workgroups go on to further blocks of rows (test_operators_choose.py: these sizes do)."""
    rows = 500_000_003
    x = torch.ones(rows, 1, 2, dtype=torch.bfloat16, device="cuda")
    r = binding.Rotary(2)
    r(x, period=1000)
    few = r(torch.ones(1000, 1, 2, dtype=torch.bfloat16, device="cuda"), period=1000)
    want, tol = _turned(torch.ones(1000, 1, 2, dtype=torch.bfloat16), np.arange(1000), 2, "half")
    _close(few, want, tol, "a period")
    whole = rows // 1000 * 1000
    assert (x[:whole].view(-1, 2000) == few.view(1, 2000)).all() and torch.equal(x[whole:], few[:rows - whole])


# ---- clipping ----

@pytest.mark.parametrize("P,sizes,kind", operator_cases.CLIP, ids=lambda v: "%dx%d" % (len(v), sum(v)) if isinstance(v, list) else str(v))
def test_clip_of_many_units_and_types(P, sizes, kind):
    """Members with norms on both sides of the bound, tensors that start at odd elements, results elsewhere and in place."""
    dtypes = [TYPES[t] for t in operator_cases.clip_dtypes(sizes, kind)]
    g = torch.Generator(device="cuda").manual_seed(P + len(sizes))
    scale = (torch.linspace(0.3, 3.0, P, device="cuda") / sum(sizes) ** 0.5)[:, None]
    grads = [(torch.randn(P, n + 1, generator=g, device="cuda") * scale).to(t)[:, 1:] for n, t in zip(sizes, dtypes)]
    outs = [torch.full((P, n + 3), 7.0, dtype=t, device="cuda")[:, 3:] for n, t in zip(sizes, dtypes)]
    norms = binding.GradClip(grads, outs)(torch.ones(1, device="cuda"))
    # (the oracle's sums in float64 on the device: the largest of these hold 130 million values)
    want_norm = torch.stack([(v.double() ** 2).sum(1) for v in grads]).sum(0).sqrt()
    factor = torch.where(want_norm > 1.0, 1.0 / want_norm, torch.ones_like(want_norm))[:, None]
    near = ((want_norm - 1.0).abs() < 1e-6)[:, None]      # (either side of the bound is right there)
    assert ((norms.double() - want_norm).abs() <= 1.01 * U * want_norm).all() and (want_norm > 1.1).any() and (P == 1 or (want_norm < 0.9).any())
    below = (want_norm < 1.0 - 1e-6)
    for v, o in zip(grads, outs):
        want = v.double() * factor
        assert (((o.double() - want).abs() <= (HALF[v.dtype] + 2.01 * U) * want.abs() + 1e-45) | near).all()
        assert torch.equal(o[below], v[below])
        assert (o._base[:, :3] == 7).all()
    again = binding.GradClip(grads)(torch.ones(1, device="cuda"))
    assert torch.equal(again, norms) and all(torch.equal(a, b) for a, b in zip(grads, outs))
