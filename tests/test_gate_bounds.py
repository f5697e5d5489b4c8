"""What csrc/activation.h says of the sigmoid's errors, in numpy's fp32 (no GPU needed): the kernels' steps, with an exponential and a reciprocal that are off by
as much as the hardware's may be, one step either way."""
import numpy as np
import pytest

f32, f64 = np.float32, np.float64
LOG2E, K = 1.4426950408889634074, 1.5957691216057307118
COEF = {"silu": (f32(LOG2E), f32(0)), "gelu": (f32(K * LOG2E), f32(K * 0.044715 * LOG2E))}
ARGUMENT = {"silu": 2.0 ** -23, "gelu": 2.0 ** -22}


def fma(a, b, c):
    """Of fp32: the product is exact in fp64, the sum there rounded once more (2^-29 of a step)."""
    return (a.astype(f64) * b + c).astype(f32)


def steps(v, n):
    return (v.view(np.int32) + n).view(f32)


def gates():
    rng = np.random.default_rng(0)
    g = np.concatenate([rng.uniform(-30, 30, 400000), rng.uniform(-1, 1, 200000), rng.uniform(-9, 9, 400000), 2.0 ** rng.uniform(-40, 6.4, 100000)])
    return g.astype(f32)


def arguments(g, act):
    """The kernel's, in units of log 2, and the exact one."""
    c0, c1 = COEF[act]
    z = g * fma(np.full_like(g, c1), g * g, c0)
    d = g.astype(f64)
    exact = LOG2E * (d if act == "silu" else K * (d + 0.044715 * d ** 3))
    return z, exact


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_argument(act):
    z, exact = arguments(gates(), act)
    off = np.abs(z - exact) / (ARGUMENT[act] * np.abs(exact))
    assert off.max() <= 1
    if act == "gelu":  # (two steps, which SiLU's argument keeps to, are not enough)
        assert off.max() > 0.55


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("de", [-1, 0, 1])
@pytest.mark.parametrize("dr", [-1, 0, 1])
def test_share(act, de, dr):
    z, exact = arguments(gates(), act)
    fine = np.abs(exact) < 120
    z, exact = z[fine], exact[fine]
    e = steps(np.exp2(-z.astype(f64)).astype(f32), 0)
    e = np.where(de != 0, np.nextafter(e, f32(np.inf if de > 0 else 0)), e)
    d = f32(1) + e
    p = (1 / d.astype(f64)).astype(f32)
    p = np.where(dr != 0, np.nextafter(p, f32(2 if dr > 0 else 0)), p)
    want = 1 / (1 + np.exp2(-exact))
    rest = 1 / (1 + np.exp2(exact))
    argument = ARGUMENT[act] * np.abs(exact) / LOG2E
    # (one step of a correctly rounded result either way is a step and a half: 2^-23 and half of it)
    assert (np.abs(p - want) <= want * (argument + 2.0 ** -21)).all()
    r = fma(-(e - (d - f32(1))), p, fma(-d, p, f32(1)))
    near = fma(p, np.clip(r, f32(-2.0 ** -20), f32(2.0 ** -20)), p)
    assert (np.abs(near - want) <= want * ((argument + 1.5 * 2.0 ** -23) * rest + 2.0 ** -24 * 1.01)).all()
