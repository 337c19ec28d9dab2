"""The operators around a step's dense products, in float64: clipping by the gradient norm, rotary positions, and the norm after a
block with its gate, the scaled residual sum and the norm before the next block (with their gradients).

  clip        n_i = sqrt(sum of squares over all tensors of member i); g <- g m_i / n_i where n_i > m_i.
  rotary      pair j of a head, elements (j, j + r/2) or (2j, 2j + 1), turns by position * f_j, f_j = base^(-2j/r); the rest of the head
              is copied.  Longer contexts: f / factor ("linear"), base * factor^(r/(r-2)) ("base"), or f (w + (1 - w) / factor) with
              w = clamp((trained f / 2 pi - low) / (high - low), 0, 1) ("ramp").  `gain` multiplies what is turned.
  block norm  u = N_post(y), out = alpha x + beta a(gate) u, z = N_pre(out); N is LayerNorm or division by the root mean square, each with
              gain and bias.
"""
import numpy as np


def clip(grads, max_norm):
    """grads: arrays [P, ...].  Returns (norms [P], clipped arrays)."""
    P = grads[0].shape[0]
    sq = sum((np.asarray(g, dtype=np.float64).reshape(P, -1) ** 2).sum(axis=1) for g in grads)
    norms = np.sqrt(sq)
    if max_norm is None:
        return norms, None
    m = np.broadcast_to(np.asarray(max_norm, dtype=np.float64), (P,))
    m = np.where(m < 0.0, 0.0, m)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(norms > m, m / norms, 1.0)
        return norms, [np.asarray(g, dtype=np.float64) * c.reshape((P,) + (1,) * (g.ndim - 1)) for g in grads]


def rotary_frequencies(rot, base=10000.0, scaling="none", factor=1.0, trained=0.0, low=1.0, high=32.0):
    """Radians a position, [rot / 2]."""
    j = np.arange(rot // 2, dtype=np.float64)
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2.0))
    f = base ** (-2.0 * j / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "ramp":
        w = np.clip((trained * f / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
        f = f * (w + (1.0 - w) / factor)
    return f


def rotary(x, positions, freq, layout="half", gain=1.0, backward=False):
    """x [rows, heads, width], positions [rows]."""
    x = np.asarray(x, dtype=np.float64)
    r = 2 * len(freq)
    # whole turns go before sine and cosine see the angle (exact: the remainder of two doubles)
    angle = np.fmod(np.asarray(positions, dtype=np.float64)[:, None] * freq, 2 * np.pi)[:, None, :]
    c, s = gain * np.cos(angle), gain * np.sin(angle) * (-1.0 if backward else 1.0)
    first, second = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    a, b = x[..., first], x[..., second]
    out = x.copy()
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    return out


def _norm(kind, v, gain, bias, eps):
    if kind == "none":
        return v, (None, None)
    if kind == "layer":
        v = v - v.mean(axis=-1, keepdims=True)
    rstd = 1.0 / np.sqrt((v * v).mean(axis=-1, keepdims=True) + eps)
    hat = v * rstd
    return hat * gain + bias, (hat, rstd)


def _norm_backward(kind, dv, gain, cache):
    if kind == "none":
        return dv
    hat, rstd = cache
    w = dv * gain
    d = w - hat * (w * hat).mean(axis=-1, keepdims=True)
    if kind == "layer":
        d = d - w.mean(axis=-1, keepdims=True)
    return rstd * d


def gate_factor(act, g):
    """(a(g), a'(g))."""
    if act == "none":
        return g, np.ones_like(g)
    if act == "tanh":
        t = np.tanh(g)
        return t, 1.0 - t * t
    with np.errstate(over="ignore"):
        s = 1.0 / (1.0 + np.exp(-g))
    return (s, s * (1.0 - s)) if act == "sigmoid" else (g * s, s * (1.0 + g * (1.0 - s)))


class BlockNorm:
    """One member: y, x, gate rows [n, d]; params: dict of [d] arrays (post_gain, post_bias, pre_gain, pre_bias, gate)."""

    def __init__(self, post="layer", pre="layer", gate="none", act="none", eps=1e-5, alpha=1.0, beta=1.0):
        self.post, self.pre, self.gate, self.act = post, pre, gate, act
        self.eps, self.alpha, self.beta = float(np.float32(eps)), float(np.float32(alpha)), float(np.float32(beta))

    def forward(self, y, x, params, gate=None):
        p = {k: np.asarray(v, dtype=np.float64) for k, v in params.items()}
        u, c1 = _norm(self.post, np.asarray(y, dtype=np.float64), p.get("post_gain", 1.0), p.get("post_bias", 0.0), self.eps)
        f, df = (1.0, 0.0) if self.gate == "none" else gate_factor(self.act, p["gate"] if self.gate == "vector" else np.asarray(gate, dtype=np.float64))
        out = self.alpha * np.asarray(x, dtype=np.float64) + self.beta * f * u
        z, c2 = _norm(self.pre, out, p.get("pre_gain", 1.0), p.get("pre_bias", 0.0), self.eps)
        return out, (None if self.pre == "none" else z), (p, u, f, df, c1, c2)

    def backward(self, cache, dout, dz):
        """(dy, dx, dgate rows or None, parameter gradients)."""
        p, u, f, df, c1, c2 = cache
        t = np.zeros_like(u) if dout is None else np.asarray(dout, dtype=np.float64)
        grads = {}
        if self.pre != "none":
            dz = np.zeros_like(u) if dz is None else np.asarray(dz, dtype=np.float64)
            t = t + _norm_backward(self.pre, dz, p.get("pre_gain", 1.0), c2)
            grads["pre_gain"], grads["pre_bias"] = (dz * c2[0]).sum(axis=0), dz.sum(axis=0)
        v = self.beta * f * t
        dgate = self.beta * df * u * t
        if self.gate == "vector":
            grads["gate"] = dgate.sum(axis=0)
        if self.post != "none":
            grads["post_gain"], grads["post_bias"] = (v * c1[0]).sum(axis=0), v.sum(axis=0)
        dy = _norm_backward(self.post, v, p.get("post_gain", 1.0), c1)
        return dy, self.alpha * t, (dgate if self.gate == "rows" else None), grads
