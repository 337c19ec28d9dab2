"""The float64 operators around the dense products: gradients against central differences, identities of the rotation, clipping."""
import numpy as np
import pytest

from oracle import operators as oo


def test_clip_scales_only_members_above_their_bound():
    rng = np.random.default_rng(0)
    grads = [rng.standard_normal((3, 5)), rng.standard_normal((3, 2, 4))]
    norms, out = oo.clip(grads, [1e-3, 1e3, 2.0])
    after, _ = oo.clip(out, None)
    assert np.allclose(norms, [np.sqrt((grads[0][i] ** 2).sum() + (grads[1][i] ** 2).sum()) for i in range(3)])
    assert np.allclose(after, np.minimum(norms, [1e-3, 1e3, 2.0])) and np.array_equal(out[0][1], grads[0][1])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_keeps_lengths_and_depends_on_distance(layout):
    rng = np.random.default_rng(1)
    f = oo.rotary_frequencies(12)
    q, k = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    turned = lambda x, p: oo.rotary(x, [p], f, layout)[0, 0]  # noqa: E731
    assert np.isclose(np.linalg.norm(turned(q, 77)), np.linalg.norm(q))
    assert np.isclose(turned(q, 5) @ turned(k, 3), turned(q, 1005) @ turned(k, 1003))
    assert np.allclose(oo.rotary(oo.rotary(q, [9], f, layout), [9], f, layout, backward=True), q)


def test_scaled_frequencies():
    f = oo.rotary_frequencies(64)
    assert np.allclose(oo.rotary_frequencies(64, scaling="linear", factor=4.0), f / 4)
    b = oo.rotary_frequencies(64, scaling="base", factor=4.0)
    assert np.isclose(b[0], f[0]) and np.isclose(b[-1], f[-1] / 4)           # the fastest keeps its pace, the slowest slows by the factor
    r = oo.rotary_frequencies(64, scaling="ramp", factor=4.0, trained=4096.0)
    assert np.isclose(r[0], f[0]) and np.isclose(r[-1], f[-1] / 4) and np.all(np.diff(r) < 0)


@pytest.mark.parametrize("post,pre", [("layer", "layer"), ("rms", "rms"), ("rms", "layer"), ("none", "rms"), ("layer", "none")])
@pytest.mark.parametrize("gate,act", [("none", "none"), ("vector", "none"), ("rows", "sigmoid"), ("rows", "silu"), ("vector", "tanh")])
def test_block_norm_gradients_against_differences(post, pre, gate, act):
    rng = np.random.default_rng(2)
    n, d = 3, 7
    b = oo.BlockNorm(post, pre, gate, act, alpha=0.9, beta=0.6)
    t = {"y": rng.standard_normal((n, d)), "x": rng.standard_normal((n, d)), "rows": rng.standard_normal((n, d))}
    params = {}
    if post != "none":
        params.update(post_gain=rng.standard_normal(d), post_bias=rng.standard_normal(d))
    if pre != "none":
        params.update(pre_gain=rng.standard_normal(d), pre_bias=rng.standard_normal(d))
    if gate == "vector":
        params["gate"] = rng.standard_normal(d)
    dout, dz = rng.standard_normal((n, d)), rng.standard_normal((n, d))

    def value():
        out, z, _ = b.forward(t["y"], t["x"], params, t["rows"])
        return (out * dout).sum() + (0.0 if z is None else (z * dz).sum())

    dy, dx, dgate, grads = b.backward(b.forward(t["y"], t["x"], params, t["rows"])[2], dout, dz)
    pairs = [(t["y"], dy), (t["x"], dx)] + [(params[k], g) for k, g in grads.items()] + ([(t["rows"], dgate)] if gate == "rows" else [])
    h = 1e-5
    for a, g in pairs:
        for at in np.ndindex(a.shape):
            keep = a[at]
            a[at] = keep + h
            up = value()
            a[at] = keep - h
            down = value()
            a[at] = keep
            # third derivatives of order 10 over h^2 = 1e-10, rounding 1e-15 / h
            assert abs((up - down) / (2 * h) - g[at]) < 1e-7 * max(1.0, abs(g[at]))
