"""Without a GPU: what the entry points on heads refuse before anything is launched, the frequencies (computed on the host), and pins of the
oracle that the kernels are compared with."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2511_23225_amd as tw
from oracle import block


@pytest.fixture(scope="module")
def memory():
    """Addresses of host memory, 256-byte aligned, 64 KB apart; nothing reads them."""
    buf = ctypes.create_string_buffer(1 << 21)
    first = (ctypes.addressof(buf) + 255) & ~255
    yield [first + i * 65536 for i in range(24)]
    del buf


def group(x, y, heads=4, dim=16, gain=None, **k):
    a = dict(x=x, y=y, x_token=heads * dim, x_head=dim, y_token=heads * dim, y_head=dim, gain=gain, heads=heads)
    a.update(k)
    return a


def call(groups, positions, freqs, name="tweo_rotary", tokens=8, dim=16, rot=16, layout=0, scale=1.0, eps=1e-6, cfg=True, count=None):
    rows = (tw.binding.Heads * max(1, len(groups)))()
    for row, g in zip(rows, groups):
        for k, v in g.items():
            setattr(row, k, v)
    c = ctypes.byref(tw.binding.RotaryCfg(positions, freqs, rot, layout, scale)) if cfg else None
    count = len(groups) if count is None else count
    lib = tw.load()
    if name == "tweo_rotary":
        return lib.tweo_rotary(rows, count, tokens, dim, c, 0, None)
    return lib.tweo_head_norm_rotary_fwd(rows, count, tokens, dim, eps, c, None)


@pytest.mark.parametrize("name", ["tweo_rotary", "tweo_head_norm_rotary_fwd"])
def test_refusals(memory, name):
    x, y, k, z, pos, f, gain = memory[:7]
    bad = lambda groups=None, **kw: call(groups or [group(x, y)], kw.pop("positions", pos), kw.pop("freqs", f), name, **kw)  # noqa: E731
    for kw in (dict(positions=None), dict(freqs=None), dict(positions=pos + 4), dict(freqs=f + 4), dict(rot=0), dict(rot=3), dict(rot=18), dict(rot=-2),
               dict(layout=2), dict(layout=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(tokens=0), dict(tokens=-1), dict(dim=0),
               dict(count=0), dict(count=3), dict(groups=[group(None, y)]), dict(groups=[group(x, None)]), dict(groups=[group(x + 1, y)]),
               dict(groups=[group(x, y + 1)]), dict(groups=[group(x, y, heads=0)]), dict(groups=[group(x, y, heads=-1)]),
               dict(groups=[group(x, y, x_token=-64)]), dict(groups=[group(x, y, y_head=-16)]),
               # overlap: of x and y by a head, of two heads of y, of two tokens of y, of both groups' outputs, of an output with the other's input
               dict(groups=[group(x, x + 32)]), dict(groups=[group(x, y, y_head=8)]), dict(groups=[group(x, y, y_head=0)]),
               dict(groups=[group(x, y, y_token=48)]), dict(groups=[group(x, y), group(k, y)]), dict(groups=[group(x, y), group(k, y + 16)]),
               dict(groups=[group(x, y), group(y, z)]), dict(groups=[group(x, x, y_token=128)]), dict(groups=[group(x, pos)]),
               dict(groups=[group(x, f - 32)])):
        assert bad(**kw) == tw.TWEO_ERR_INVALID_ARG, kw
    for kw in (dict(dim=513), dict(tokens=(1 << 30) + 1), dict(groups=[group(x, y, heads=65537)]),
               dict(groups=[group(x, y, heads=1 << 16)], tokens=1 << 20), dict(groups=[group(x, y, x_token=1 << 45)])):
        assert bad(**kw) == tw.TWEO_ERR_UNSUPPORTED, kw
    if name == "tweo_rotary":
        assert bad(cfg=False) == tw.TWEO_ERR_INVALID_ARG
        assert bad(groups=[group(x, y, gain=gain)]) == tw.TWEO_ERR_INVALID_ARG
        assert tw.load().tweo_rotary(None, 1, 8, 16, ctypes.byref(tw.binding.RotaryCfg(pos, f, 16, 0, 1.0)), 0, None) == tw.TWEO_ERR_INVALID_ARG
    else:
        for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(groups=[group(x, y, gain=gain + 1)]), dict(groups=[group(x, y, gain=y)])):
            assert bad(**kw) == tw.TWEO_ERR_INVALID_ARG, kw


def test_heads_of_one_tensor_that_overlap(memory):
    """Queries and keys side by side in a qkv tensor, in place, or interleaved head by head, a little off their places (where they are right: on the GPU)."""
    x, pos, f = memory[0], memory[2], memory[3]
    clash = lambda *groups: call(list(groups), pos, f, rot=16) == tw.TWEO_ERR_INVALID_ARG  # noqa: E731
    assert clash(group(x, x, x_token=192, y_token=192), group(x + 120, x + 120, x_token=192, y_token=192))      # eight bytes too early
    assert clash(group(x, x, x_token=192, y_token=192), group(x + 288, x + 288, x_token=192, y_token=192))      # into the next token
    assert clash(group(x, x, x_head=32, y_head=32, x_token=128, y_token=128), group(x + 16, x + 16, x_head=32, y_head=32, x_token=128, y_token=128))


def grad_group(dy, x, dx, heads=4, dim=16, gain=None, dgain=None, **k):
    a = dict(dy=dy, x=x, dx=dx, dy_token=heads * dim, dy_head=dim, x_token=heads * dim, x_head=dim, dx_token=heads * dim, dx_head=dim, gain=gain,
             dgain=dgain, heads=heads)
    a.update(k)
    return a


def test_grad_refusals(memory):
    dy, x, dx, gain, dgain, pos, f, ws = memory[:8]
    lib = tw.load()

    def bwd(groups=None, tokens=8, dim=16, rot=16, eps=1e-6, ws=ws, n=1 << 16, cfg=True, count=None):
        groups = [grad_group(dy, x, dx, gain=gain, dgain=dgain)] if groups is None else groups
        rows = (tw.binding.HeadsGrad * max(1, len(groups)))()
        for row, g in zip(rows, groups):
            for k, v in g.items():
                setattr(row, k, v)
        c = ctypes.byref(tw.binding.RotaryCfg(pos, f, rot, 0, 1.0)) if cfg else None
        return lib.tweo_head_norm_rotary_bwd(rows, len(groups) if count is None else count, tokens, dim, eps, c, ws, n, None)

    G = lambda **k: [grad_group(**{**dict(dy=dy, x=x, dx=dx, gain=gain, dgain=dgain), **k})]  # noqa: E731
    for kw in (dict(groups=G(dy=None)), dict(groups=G(x=None)), dict(groups=G(dx=None)), dict(groups=G(dy=dy + 1)), dict(groups=G(x=x + 1)),
               dict(groups=G(dx=dx + 1)), dict(groups=G(gain=gain + 1)), dict(groups=G(dgain=dgain + 4)), dict(groups=G(heads=0)), dict(tokens=0),
               dict(dim=0), dict(rot=5), dict(rot=32), dict(eps=-1.0), dict(eps=float("nan")), dict(count=0), dict(count=3), dict(groups=G(dx=dy + 32)),
               dict(groups=G(dx=x + 32)), dict(groups=G(dx=dgain)), dict(groups=G(dx=ws)), dict(groups=G(dgain=ws)), dict(groups=G(dx=gain)),
               dict(groups=G(dx_head=8)), dict(groups=G(dy_token=-1)), dict(groups=G() + G(dgain=dgain))):
        assert bwd(**kw) == tw.TWEO_ERR_INVALID_ARG, kw
    for kw in (dict(dim=513), dict(tokens=(1 << 30) + 1), dict(groups=G(heads=65537))):
        assert bwd(**kw) == tw.TWEO_ERR_UNSUPPORTED, kw
    need = tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, 8, 4, 16)
    assert need >= 256 and need % 256 == 0
    for kw in (dict(ws=None), dict(ws=ws + 8), dict(n=0), dict(n=8 * 4 * 16 * 4 - 1)):
        assert bwd(**kw) == tw.TWEO_ERR_WORKSPACE, kw
    assert lib.tweo_head_norm_rotary_bwd(None, 1, 8, 16, 1e-6, None, ws, 1 << 16, None) == tw.TWEO_ERR_INVALID_ARG
    # a row for each of some 1400 workgroups at most, whatever the sizes
    assert tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, 1 << 30, 1 << 17, 512) <= 1500 * 512 * 4
    assert tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, 1 << 62, 1 << 62, 1 << 62) <= 1500 * 512 * 4


def test_frequencies():
    f = tw.tweo_rotary_freqs(128)
    assert f.dtype is torch.float64 and f.device.type == "cpu"
    want = np.array([math.exp(-2 * i / 128 * math.log(10000.0)) for i in range(64)])
    assert np.allclose(f.numpy(), want, rtol=1e-14, atol=0)
    assert np.allclose(tw.tweo_rotary_freqs(96, base=500000.0).numpy(), 500000.0 ** (-np.arange(48) / 48), rtol=1e-14, atol=0)
    assert np.allclose(tw.tweo_rotary_freqs(128, kind="linear", factor=4.0).numpy(), want / 4, rtol=1e-14, atol=0)
    based = tw.tweo_rotary_freqs(128, kind="base", factor=8.0).numpy()
    assert based[0] == 1.0 and np.isclose(based[-1], want[-1] / 8, rtol=1e-13, atol=0) and (np.diff(based) < 0).all()
    t = tw.tweo_rotary_freqs(128, kind="turns", factor=4.0, context=8192, low_turns=1, high_turns=32).numpy()
    n = 8192 * want / (2 * math.pi)
    assert (t[n >= 32] == f.numpy()[n >= 32]).all() and np.allclose(t[n <= 1], want[n <= 1] / 4, rtol=1e-14, atol=0)
    mid = (n > 1) & (n < 32)
    s = (n[mid] - 1) / 31
    assert mid.any() and np.allclose(t[mid], want[mid] * (s + (1 - s) / 4), rtol=1e-13, atol=0)
    good = dict(rot_dim=16, base=10000.0, factor=2.0, context=100.0, low_turns=1.0, high_turns=2.0)
    for k in (dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=-2), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")),
              dict(kind="linear", factor=0.5), dict(kind="linear", factor=float("nan")), dict(kind="base", rot_dim=2), dict(kind="turns", context=0.0),
              dict(kind="turns", low_turns=2.0), dict(kind="turns", low_turns=-1.0), dict(kind="turns", high_turns=float("inf"))):
        with pytest.raises(tw.TweoError) as e:
            tw.tweo_rotary_freqs(**{**good, **k})
        assert e.value.status == tw.TWEO_ERR_INVALID_ARG, k
    with pytest.raises(ValueError):
        tw.tweo_rotary_freqs(16, kind="other")


# ---- the oracle
def test_oracle_rotation_is_one():
    rng = np.random.default_rng(0)
    x, f = rng.standard_normal((6, 3, 20)), 100.0 ** (-np.arange(6) / 6)
    pos = np.array([0, 1, 5, 1000, 7, 2])
    for layout in ("halves", "pairs"):
        y, _ = block.rotary(x, pos, f, layout)
        assert np.allclose(y[0], x[0]) and (y[..., 12:] == x[..., 12:]).all()
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        back, _ = block.rotary(y, pos, f, layout, transpose=True)
        assert np.allclose(back, x)
        # a product of a query and a key depends on the distance alone
        q, k = x[0, 0], x[1, 1]
        dots = [(block.rotary(q[None, None], [p], f, layout)[0] * block.rotary(k[None, None], [p + 3], f, layout)[0]).sum() for p in (0, 4, 11)]
        assert np.allclose(dots, dots[0])
    # the members of a pair, as complex numbers
    z = x[..., :6] + 1j * x[..., 6:12]
    y, _ = block.rotary(x, pos, f, "halves", scale=1.5)
    want = 1.5 * z * np.exp(1j * pos[:, None] * f)[:, None]
    assert np.allclose(y[..., :6], want.real) and np.allclose(y[..., 6:12], want.imag)


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_oracle_gradients_against_differences(layout):
    rng = np.random.default_rng(1)
    x, gain, dy = rng.standard_normal((3, 2, 10)), 1 + 0.2 * rng.standard_normal(10), rng.standard_normal((3, 2, 10))
    args = (1e-3, [3, 0, 7], 50.0 ** (-np.arange(4) / 4), layout, 1.25)
    loss = lambda x, gain: (dy * block.head_norm_rotary(x, gain, *args)[0]).sum()  # noqa: E731
    dx, dgain, _, _ = block.head_norm_rotary_bwd(dy, x, gain, *args)
    h = 1e-6
    for at in [(0, 0, 0), (1, 1, 3), (2, 0, 9), (2, 1, 6)]:
        step = np.zeros_like(x)
        step[at] = h
        assert np.isclose((loss(x + step, gain) - loss(x - step, gain)) / (2 * h), dx[at], rtol=1e-6, atol=1e-8)
    for i in range(10):
        step = np.zeros_like(gain)
        step[i] = h
        assert np.isclose((loss(x, gain + step) - loss(x, gain - step)) / (2 * h), dgain[i], rtol=1e-6, atol=1e-8)
