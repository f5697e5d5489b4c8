"""LayerNorm's gradients, the gradients' norm and AdamW in numpy, fp64 except where the method fixes the type.

TEST INFRASTRUCTURE ONLY, like the rest of this package; shares no code with the product.
"""
import numpy as np


def layernorm_stats(h, eps):
    """(mean, 1 / sqrt(var + eps)) of each row, fp64 [rows, 2]."""
    mean = h.mean(1)
    with np.errstate(all="ignore"):
        return np.stack([mean, 1.0 / np.sqrt(((h - mean[:, None]) ** 2).mean(1) + eps)], 1)


def layernorm_bwd(dy, h, gamma, stats, dres=None):
    """dx, dgamma, dbeta, and what bounds the error of an fp32 evaluation: the sums of the magnitudes of their terms."""
    with np.errstate(all="ignore"):
        rstd = stats[:, 1:]
        xhat = (h - stats[:, :1]) * rstd
        w = dy * gamma
        c1, c2 = (w * xhat).mean(1, keepdims=True), w.mean(1, keepdims=True)
        dx = rstd * (w - c2 - xhat * c1)
        size = rstd * (np.abs(w) + np.abs(w).mean(1, keepdims=True) + np.abs(xhat) * np.abs(w * xhat).mean(1, keepdims=True))
        if dres is not None:
            dx, size = dx + dres, size + np.abs(dres)
        return dx, (dy * xhat).sum(0), dy.sum(0), size, np.abs(dy * xhat).sum(0), np.abs(dy).sum(0)


def clip_factor(sumsq, max_norm):
    return min(1.0, max_norm / (np.sqrt(sumsq) + 1e-6))


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, decay, clip=1.0):
    """New p, m, v in fp64, and the sizes of the terms of m and of the change of p."""
    g = g * clip
    m1 = beta1 * m + (1 - beta1) * g
    v1 = beta2 * v + (1 - beta2) * g * g
    denom = np.sqrt(v1 / (1 - beta2 ** t)) + eps
    rate = lr / (1 - beta1 ** t)
    m_size = beta1 * np.abs(m) + (1 - beta1) * np.abs(g)
    with np.errstate(all="ignore"):
        p1 = p - lr * decay * p - rate * m1 / denom
        return p1, m1, v1, m_size, rate * m_size / denom + lr * decay * np.abs(p)


FORMATS = {"e4m3": dict(top=448.0, mantissa=3, least=-6, largest=0x7E, bias=7), "e5m2": dict(top=57344.0, mantissa=2, least=-14, largest=0x7B, bias=15)}


def decode(codes, fmt):
    f = FORMATS[fmt]
    b = codes.astype(np.int64)
    e, frac = (b & 0x7F) >> f["mantissa"], (b & ((1 << f["mantissa"]) - 1)) / 2.0 ** f["mantissa"]
    mag = np.where(e > 0, (1 + frac) * 2.0 ** (e - f["bias"]), frac * 2.0 ** (1 - f["bias"]))
    return np.where(b & 0x80, -mag, mag)


def threshold(n, t, fmt):
    """u of the elements 0 .. n - 1 at step t, as its top bits."""
    w = (np.arange(n, dtype=np.uint64) * np.uint64(0x6A09E667) + np.uint64(t) * np.uint64(0x9E3779B9)) & np.uint64(0xFFFFFFFF)
    bits = 23 - FORMATS[fmt]["mantissa"]
    return (w >> np.uint64(32 - bits)).astype(np.float64) / 2.0 ** bits


def encode(x, t, fmt):
    """Codes (magnitudes with sign), steps and the distance of each element from where its code would change, for fp32 values x: the
    scales are single fp32 divisions of a block of 256, the scaled value one fp32 product, the rest exact."""
    f = FORMATS[fmt]
    x = x.astype(np.float32)
    pad = np.zeros(-x.size % 256, np.float32)
    blocks = np.abs(np.concatenate([x, pad])).reshape(-1, 256)
    amax = blocks.max(1)
    with np.errstate(all="ignore"):
        scale = np.where(amax > 0, np.minimum(np.float32(f["top"]) / amax, np.finfo(np.float32).max), np.float32(1)).astype(np.float32)
        step = np.float32(1) / scale
    y = (blocks * scale[:, None]).reshape(-1)[:x.size].astype(np.float64)
    _, e = np.frexp(y)
    unit = 2.0 ** (np.maximum(e - 1, f["least"]) - f["mantissa"])
    # a value that lies that far below the normal codes is first rounded to 2^-20 (2^-21) of its unit, to even
    fine = 2.0 ** (23 - f["mantissa"])
    at = np.rint(y / unit * fine) / fine + threshold(x.size, t, fmt)
    whole = np.floor(at)
    value = np.minimum(whole * unit, f["top"])
    if fmt == "e5m2":  # a positive second moment stays positive
        value = np.where((value == 0) & (x > 0), 2.0 ** -16, value)
    return value, step, np.abs(at - np.rint(at)), unit
