"""What a block runs between its linears - rotary positions, norms of heads, the gated feed-forward - in numpy, fp64.

TEST INFRASTRUCTURE ONLY, like the rest of this package; shares no code with the product.
"""
import numpy as np


def turns(positions, freqs):
    """Cosines and sines of position * frequency, [tokens, pairs].  (The product in extended precision, so that far positions keep their angle.)"""
    angle = np.asarray(positions, np.longdouble)[:, None] * np.asarray(freqs, np.longdouble)
    return np.cos(angle).astype(np.float64), np.sin(angle).astype(np.float64)


def _members(rot, layout):
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if layout == "halves" else (2 * i, 2 * i + 1)


def rotary(x, positions, freqs, layout="halves", scale=1.0, transpose=False):
    """x [tokens, heads, dim]; also what bounds an fp32 evaluation: the sums of the magnitudes of each result's terms."""
    y, size = x.copy(), np.abs(x)
    if freqs is None:
        return y, size
    c, s = turns(positions, freqs)
    s = -s if transpose else s
    i, j = _members(2 * len(freqs), layout)
    c, s = c[:, None], s[:, None]
    with np.errstate(invalid="ignore"):
        a, b = x[..., i], x[..., j]
        y[..., i], y[..., j] = scale * (a * c - b * s), scale * (b * c + a * s)
    size[..., i] = size[..., j] = abs(scale) * (np.abs(a) + np.abs(b))
    return y, size


def head_norm(x, gain, eps):
    """x * rstd * gain over the last index."""
    with np.errstate(all="ignore"):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain


def head_norm_rotary(x, gain, eps, positions=None, freqs=None, layout="halves", scale=1.0):
    return rotary(head_norm(x, gain, eps), positions, freqs, layout, scale)


def head_norm_rotary_bwd(dy, x, gain, eps, positions=None, freqs=None, layout="halves", scale=1.0):
    """dx, dgain and the sums of the magnitudes of their terms."""
    d, size = rotary(dy, positions, freqs, layout, scale, transpose=True)
    with np.errstate(all="ignore"):
        rstd = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        xhat = x * rstd
        w, ws = d * gain, size * np.abs(gain)
        dx = rstd * (w - xhat * (w * xhat).mean(-1, keepdims=True))
        dx_size = rstd * (ws + np.abs(xhat) * (ws * np.abs(xhat)).mean(-1, keepdims=True))
        return dx, (d * xhat).sum((0, 1)), dx_size, (size * np.abs(xhat)).sum((0, 1))


GELU = np.sqrt(2 / np.pi), 0.044715


def gate_argument(g, act):
    """z and dz/dg of act(g) = g * sigmoid(z): g itself, or, as 1 + tanh(y) = 2 sigmoid(2y), twice the tanh form's argument."""
    return (g, np.ones_like(g)) if act == "silu" else (2 * GELU[0] * (g + GELU[1] * g ** 3), 2 * GELU[0] * (1 + 3 * GELU[1] * g * g))


def activation(g, act):
    with np.errstate(all="ignore"):
        return g / (1 + np.exp(-gate_argument(g, act)[0]))


def activation_slope(g, act):
    with np.errstate(all="ignore"):
        z, dz = gate_argument(g, act)
        p, rest = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z))
        return p + np.where(p * rest == 0, 0.0, g * p * rest * dz)
