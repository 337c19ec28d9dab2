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


# ---- inside the transformer workload ----

def _fd_network(h=(1e-3, 0.0, 0.0), **options):
    from oracle import transformer as tf
    spec = tf.TransformerSpec(vocab=11, d_model=8, n_heads=2, d_ff=12, n_layers=2, seq=5, batch=2, seed=3, **options)
    rng = np.random.default_rng(4)
    arrays = [1.0 + 0.2 * rng.standard_normal(s) if "_g" in n else 0.4 * rng.standard_normal(s) for n, s in spec.param_shapes()]
    m = tf.new_member(spec, arrays, h, 0)
    seqs = rng.integers(0, 11, (2, 6))
    loss, grads = tf.loss_and_grads(spec, m, seqs, 1, 0)
    e = 1e-6
    for arr, g, (name, _) in zip(m.theta, grads, spec.param_shapes()):
        at = list(np.ndindex(*arr.shape))
        for k in rng.choice(len(at), size=min(6, len(at)), replace=False):
            keep = arr[at[k]]
            arr[at[k]] = keep + e
            up = tf.loss_and_grads(spec, m, seqs, 1, 0)[0]
            arr[at[k]] = keep - e
            down = tf.loss_and_grads(spec, m, seqs, 1, 0)[0]
            arr[at[k]] = keep
            # (rounding of a loss of about 3 over 2e-6: 5e-10; third derivatives times 1e-12)
            assert abs((up - down) / (2 * e) - g[at[k]]) <= 2e-6 * max(1.0, abs(g[at[k]])), (name, at[k])
    return spec, m, loss


@pytest.mark.parametrize("options", [
    dict(rotary=dict(rot_dim=4)), dict(rotary=dict(rot_dim=2, layout="interleaved", gain=1.3), learned_positions=False),
    dict(block_norm="layer", alpha=0.9, beta=0.6), dict(block_norm="rms", rotary=dict(rot_dim=4, scaling="linear", factor=2.0), learned_positions=False)],
    ids=lambda o: "-".join(o))
@pytest.mark.parametrize("drop", [0.0, 0.3])
def test_transformer_with_options_against_differences(options, drop):
    _fd_network(h=(1e-3, drop, 0.1), **options)


def test_transformer_without_positions_sees_only_a_causal_bag():
    """With neither learned nor rotary positions the last position's logits do not depend on the order of the tokens before it; with rotary ones they do."""
    from oracle import transformer as tf
    rng = np.random.default_rng(5)
    for rotary, same in ((None, True), (dict(rot_dim=4), False)):
        spec = tf.TransformerSpec(vocab=11, d_model=8, n_heads=2, d_ff=12, n_layers=1, seq=5, batch=1, seed=3, learned_positions=False, rotary=rotary)
        arrays = [1.0 + 0.1 * rng.standard_normal(s) if "_g" in n else 0.5 * rng.standard_normal(s) for n, s in spec.param_shapes()]
        P = tf.params_of(spec, tf.new_member(spec, arrays, (1e-3, 0, 0), 0))
        drop = tf._Drop(spec, 0, 0, 0.0, False)
        a = tf.forward(spec, P, np.array([[1, 2, 3, 4, 5]]), drop)[0][-1]
        b = tf.forward(spec, P, np.array([[3, 1, 4, 2, 5]]), drop)[0][-1]
        assert np.allclose(a, b) == same


def test_clipped_update_uses_the_scaled_gradient():
    from oracle import optim
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    assert optim.clip(g, 10.0) is g
    assert np.allclose(np.concatenate([a.ravel() for a in optim.clip(g, 1.0)]), [0.6, 0.0, 0.8])
    assert not np.concatenate([a.ravel() for a in optim.clip(g, -1.0)]).any()
