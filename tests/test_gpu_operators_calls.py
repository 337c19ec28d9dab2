"""Calls of the operators that their documentation allows, on streams, on memory that is shared or laid out otherwise, and those that are refused."""
import copy
import pickle

import numpy as np
import pytest
import torch

from oracle import operators as oo
from paper_1711_09846_amd import binding
from tests.test_gpu_operators import CHAIN, _case, _close, _cpu, _magnitudes

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _gen(seed=0):
    return torch.Generator().manual_seed(seed)


def _normal(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def test_rotary_dropped_while_a_call_on_another_stream_is_pending():
    """The table's memory is not given away before that call has read it."""
    x = _normal(_gen(1), 64, 2, 64)
    want = binding.Rotary(64)(x, torch.empty_like(x), start=5)
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    r = binding.Rotary(64)
    table = r.table.data_ptr()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)      # (some 50 ms)
        r(x, out, start=5)
    del r
    others = [torch.zeros(32, dtype=torch.float64, device="cuda") for _ in range(64)]
    assert not side.query() and table not in [t.data_ptr() for t in others]
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_clip_of_tensors_that_meet_is_refused():
    """One tensor's result over another's gradient; norms alone may be taken of them."""
    a, b, c = (torch.ones(2, 40, device="cuda") for _ in range(3))
    bound = torch.ones(2, device="cuda")
    for grads, outs in (([a, b], [c, a]), ([a, a[:, :8]], [a, b[:, :8]]), ([a[:, :20], a[:, 19:]], None)):
        clip = binding.GradClip(grads, outs)
        with pytest.raises(binding.PbtError, match="overlap"):
            clip(bound)
        assert clip().shape == (2,)
    assert all((t == 1).all() for t in (a, b, c))
    # the same gradient into two places is fine
    binding.GradClip([a, a], [b, c])(bound)
    assert torch.equal(b, c) and (b < 1).all()


def test_clip_norms_over_the_bounds_are_refused():
    """The bounds are read by workgroups that other members' norms do not wait for."""
    a = torch.ones(2, 40, device="cuda")
    bound = torch.ones(2, device="cuda")
    with pytest.raises(binding.PbtError, match="norm"):
        binding.GradClip([a])(bound, norms=bound)
    both = torch.ones(2, 2, device="cuda")
    assert binding.GradClip([a])(both[0], norms=both[1]) is not None and (both[0] == 1).all()
    # bounds in a column beside the gradients in one array
    store = torch.ones(3, 64, device="cuda")
    norms = binding.GradClip([store[:, 1:64]])(store[:, 0])
    assert torch.equal(norms, torch.full_like(norms, 63.0 ** 0.5)) and (store[:, 0] == 1).all() and (store[:, 1:] < 0.2).all()


def test_block_norm_gradients_into_one_tensor_are_refused():
    """Two parameters' gradients into the same memory, or over a parameter; columns of one store are fine."""
    P, rows, d = 2, 6, 40
    g = _gen(2)
    y, x, dout, dz = (_normal(g, P * rows, d) for _ in range(4))
    params = dict(post_gain=1 + _normal(g, P, d, scale=0.1), pre_gain=1 + _normal(g, P, d, scale=0.1))
    op = binding.BlockNorm(d, members=P)
    _, _, stats = op.forward(y, x, params)
    _, _, _, want = op.backward(y, x, params, stats, dout, dz)
    one = torch.zeros(P, d, device="cuda")
    for grads in (dict(post_gain=one, pre_gain=one), dict(post_gain=one, pre_gain=params["pre_gain"])):
        with pytest.raises(binding.PbtError, match="overlaps"):
            op.backward(y, x, params, stats, dout, dz, grads=grads)
    store = torch.zeros(P, 100, device="cuda")
    grads = dict(post_gain=store[:, 1:41], pre_gain=store[:, 41:81])
    op.backward(y, x, params, stats, dout, dz, grads=grads)
    assert all(torch.equal(grads[k], want[k]) for k in want) and not store[:, 0].any() and not store[:, 81:].any()
    with pytest.raises(binding.PbtError, match="overlaps"):
        op.forward(y, x, params, out=x, z=x)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("order", ["head-part", "row-outermost-padded", "heads-outermost"])
def test_rotary_of_query_and_key_heads_that_lie_side_by_side(dtype, order):
    """A joint projection with a head's query, key and value next to one another: both turned in place in one call, values as they were."""
    rows, heads, w = 33, 5, 24
    g = _gen(4)
    if order == "heads-outermost":
        joint = _normal(g, heads, rows, 3, w, dtype=dtype).transpose(0, 1)
    elif order == "head-part":
        joint = _normal(g, rows, heads, 3, w, dtype=dtype)
    else:
        joint = _normal(g, rows, heads * 3 * w + 7, dtype=dtype)[:, 3:3 + heads * 3 * w].unflatten(1, (heads, 3, w))
    keep = joint.clone()
    r = binding.Rotary(18)
    q, k = joint[:, :, 0], joint[:, :, 1]
    want = [r(t, torch.empty(rows, heads, w, dtype=dtype, device="cuda"), start=3) for t in (q, k)]
    r([q, k], start=3)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(joint[:, :, 2], keep[:, :, 2])
    # from queries into the place of the values
    back = r(q, torch.empty(rows, heads, w, dtype=dtype, device="cuda"), start=3, backward=True)
    r(q, joint[:, :, 2], start=3, backward=True)
    assert torch.equal(q, want[0]) and torch.equal(joint[:, :, 2], back) and torch.equal(k, want[1])
    # half of a query and half of a key
    if order == "head-part":
        flat = joint.flatten(1)
        with pytest.raises(binding.PbtError, match="overlaps"):
            r([q, flat[:, w // 2:w // 2 + heads * 3 * w - 2 * w].unfold(1, w, 3 * w)], start=3)


def test_calls_that_would_lose_a_graph_are_refused():
    """Under gradient mode a tensor that requires a gradient is refused; without it, and inside an autograd.Function, it is not."""
    x = torch.randn(6, 2, 8, generator=_gen(5)).cuda()
    leaf = x.clone().requires_grad_()
    r = binding.Rotary(8)
    empty = lambda: torch.empty(6, 2, 8, device="cuda")  # noqa: E731
    for src, dst in ((leaf, empty()), ([x, leaf], [empty(), empty()]), (x, leaf), (leaf * 2, empty())):
        with pytest.raises(ValueError, match="graph"):
            r(src, dst)

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, t):
            return r(t, torch.empty_like(t), start=3)

        @staticmethod
        def backward(ctx, g):
            return r(g.contiguous(), torch.empty_like(g), start=3, backward=True)

    w = torch.randn(6, 2, 8, generator=_gen(6)).cuda()
    (Turn.apply(leaf) * w).sum().backward()
    with torch.no_grad():
        assert torch.equal(leaf.grad, r(w, torch.empty_like(w), start=3, backward=True))
        r(leaf, empty())

    y, h, gain = torch.randn(6, 16, generator=_gen(7)).cuda(), torch.randn(6, 16, generator=_gen(8)).cuda(), torch.ones(16, device="cuda")
    op = binding.BlockNorm(16)
    want = op.forward(y, h, dict(pre_gain=gain))
    for args in ((y.clone().requires_grad_(), h, {}), (y, h.clone().requires_grad_(), {}), (y, h, dict(pre_gain=gain.clone().requires_grad_()))):
        with pytest.raises(ValueError, match="graph"):
            op.forward(*args)
        with torch.no_grad():
            op.forward(*args)
    # gradients are what backward hands out itself
    param = dict(pre_gain=gain.clone().requires_grad_())
    grads = op.backward(y, h, param, want[2], h, y)[3]
    assert grads["pre_gain"].shape == (1, 16) and not grads["pre_gain"].requires_grad


def test_tensors_that_calls_write_are_marked_as_written():
    """A graph that saved one of them says so in its backward pass instead of using the new values."""
    rows, d = 6, 16
    store = torch.ones(1, 4 * d, device="cuda")
    g = _gen(9)

    def saved(t, write):
        w = torch.ones_like(t, requires_grad=True)
        (w * t).sum().backward()             # (untouched: fine)
        y = (w * t).sum()
        write()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()

    x = _normal(g, rows, 2, 8)
    r = binding.Rotary(8)
    saved(x, lambda: r(x, start=1))
    other = _normal(g, rows, 2, 8)
    saved(other, lambda: r([x, x.clone()], [torch.empty_like(x), other], start=1))
    grad, bound = _normal(g, 2, 40), torch.full((2,), 1e-3, device="cuda")
    clip = binding.GradClip([grad, torch.ones(2, d, device="cuda")])
    saved(grad, lambda: clip(bound))
    norms = torch.empty(2, device="cuda")
    saved(norms.zero_(), lambda: clip(norms=norms))
    columns = binding.GradClip([store[:, :d], store[:, d:2 * d]])
    saved(store, lambda: columns(bound[:1]))
    y, h, dout, dz = (_normal(g, rows, d) for _ in range(4))
    op = binding.BlockNorm(d)
    stats = op.forward(y, h)[2]
    dy, dx, gain = torch.zeros_like(y), torch.zeros_like(h), torch.zeros(1, d, device="cuda")
    params = dict(pre_gain=torch.ones(1, d, device="cuda"))
    for t in (dy, dx, gain):
        saved(t, lambda: op.backward(y, h, params, stats, dout, dz, dy=dy, dx=dx, grads=dict(pre_gain=gain)))
    saved(h, lambda: op.forward(y, h, out=h))
    saved(y, lambda: op.forward(y, h, z=y))
    # what is read only stays usable
    w = torch.ones_like(dout, requires_grad=True)
    out = (w * dout).sum()
    op.backward(y, h, {}, stats, dout, dz)
    clip()
    out.backward()
    assert torch.equal(w.grad, dout)
    with torch.inference_mode():
        t = torch.ones(3, 1, 8, device="cuda")
        r(t)
    r(t)


def test_block_norm_backward_without_statistics_is_refused():
    y = torch.zeros(2, 16, device="cuda")
    op = binding.BlockNorm(16)
    stats = op.forward(y, y, stats=False)[2]
    with pytest.raises(ValueError, match="stats"):
        op.backward(y, y, {}, stats, y, y)


@pytest.mark.parametrize("act,far", [("tanh", 12.0), ("sigmoid", 22.0), ("silu", 22.0)])
@pytest.mark.parametrize("gate", ["rows", "vector"])
def test_block_norm_gradients_of_saturated_gates(gate, act, far):
    """A gate's slope keeps its relative precision where the gate is nearly 0 or 1 (the float64 oracle's own does as far as is looked at here: 1 - tanh(12)^2 is
    1.5e-10).  dgate = beta a'(g) u t, the rest of it as in test_gpu_operators.py.  a'(g): by at most 16 U of itself (silu: of s (1 + |g| (1 - s)), its terms); tanh:
    the exponent 2 |g| log2 e is off by the roundings of its constant and its product, 2 U of itself, which moves the exponential by 4 |g| U of itself."""
    rows, d = 40, 64
    kw = dict(post="rms", pre="rms", gate=gate, act=act, dtype="fp32", res="fp32")
    c = _case(1, rows, d, **kw)
    g = torch.linspace(-far, far, rows * d if gate == "rows" else d).cuda()
    if gate == "rows":
        c["gate"] = g.view(rows, d)
    else:
        c["params"]["gate"] = g.view(1, d)
    op, spec = binding.BlockNorm(d, post="rms", pre="rms", gate=gate, act=act, alpha=0.9, beta=0.7), oo.BlockNorm("rms", "rms", gate, act, alpha=0.9, beta=0.7)
    _, _, stats = op.forward(c["y"], c["x"], c["params"], gate=c["gate"])
    _, _, dgate, grads = op.backward(c["y"], c["x"], c["params"], stats, c["dout"], c["dz"], gate=c["gate"])
    p = {k: _cpu(v[0]) for k, v in c["params"].items()}
    arrays = [None if c[k] is None else _cpu(c[k]) for k in ("y", "x", "gate", "dout", "dz")]
    w = spec.backward(spec.forward(arrays[0], arrays[1], p, arrays[2])[2], arrays[3], arrays[4])
    m = _magnitudes(spec, arrays[0], arrays[1], p, *arrays[2:])
    got, want, mag = (dgate, w[2], m["dgate"]) if gate == "rows" else (grads["gate"][0], w[3]["gate"], m["gate"])
    tol = (1.01 * CHAIN + 16 + (rows if gate == "vector" else 0) + (4 * np.abs(_cpu(g)).reshape(mag.shape) if act == "tanh" else 0)) * U * mag
    if act == "silu":
        gn = _cpu(g)
        s = 1.0 / (1.0 + np.exp(-gn))
        slope = np.abs(s * (1.0 + gn * (1.0 - s)))
        tol = tol * np.maximum(1.0, s * (1.0 + np.abs(gn) * (1.0 - s)) / np.maximum(slope, 1e-30)).reshape(mag.shape)
    _close(got, want, tol, act)


@pytest.mark.parametrize("how", [copy.deepcopy, lambda o: pickle.loads(pickle.dumps(o))], ids=["deepcopy", "pickle"])
def test_copies_of_plans(how):
    """Rotary and BlockNorm hold settings and a table: a copy of a model that has them works like the model."""
    x = _normal(_gen(3), 6, 2, 32)
    r, op = binding.Rotary(32, base=500.0), binding.BlockNorm(64, post="rms", pre="rms")
    y = x.view(6, 64)
    want = r(x, torch.empty_like(x), start=2), op.forward(y, y)[1]
    r2, op2 = how(r), how(op)
    assert r2.table.data_ptr() != r.table.data_ptr()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = r2(x, torch.empty_like(x), start=2), op2.forward(y, y)[1]
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
