"""Without a GPU: what the norm and optimizer entry points refuse before anything is launched, and pins of the oracle they are compared with."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2511_23225_amd as tw
from oracle import training


@pytest.fixture(scope="module")
def lib():
    return tw.load()


@pytest.fixture(scope="module")
def memory():
    """Addresses of host memory, 16-byte aligned, 64 KB apart; nothing reads them."""
    buf = ctypes.create_string_buffer(1 << 21)
    first = (ctypes.addressof(buf) + 255) & ~255
    yield [first + i * 65536 for i in range(24)]
    del buf


def test_layernorm_refusals(lib, memory):
    x, r, g, b, h, y, st, ws = memory[:8]
    good = dict(x=x, r=None, g=g, b=None, rows=4, cols=16, eps=1e-5, h=None, y=y, st=None)

    def fwd(**k):
        a = {**good, **k}
        return lib.tweo_layernorm_fwd(a["x"], a["r"], a["g"], a["b"], a["rows"], a["cols"], a["eps"], a["h"], a["y"], a["st"], None)

    for k in (dict(x=None), dict(y=None), dict(g=None), dict(rows=0), dict(cols=-1), dict(x=x + 2), dict(y=y + 8), dict(g=g + 2), dict(b=b + 2),
              dict(st=st + 8), dict(eps=-1.0), dict(eps=float("nan")), dict(r=r), dict(r=r, h=y), dict(r=r + 2, h=h), dict(r=r, h=h + 2)):
        assert fwd(**k) == tw.TWEO_ERR_INVALID_ARG, k
    for k in (dict(rows=(1 << 30) + 1), dict(cols=(1 << 24) + 1)):
        assert fwd(**k) == tw.TWEO_ERR_UNSUPPORTED, k
    good = dict(dy=x, h=h, g=g, st=st, dres=None, rows=4, cols=16, dx=y, dg=r, db=None, ws=ws, n=1 << 16)

    def bwd(**k):
        a = {**good, **k}
        return lib.tweo_layernorm_bwd(a["dy"], a["h"], a["g"], a["st"], a["dres"], a["rows"], a["cols"], a["dx"], a["dg"], a["db"], a["ws"], a["n"], None)

    for k in (dict(dy=None), dict(h=None), dict(g=None), dict(st=None), dict(dx=None), dict(dg=None), dict(rows=0), dict(cols=0), dict(dy=x + 2),
              dict(h=h + 2), dict(st=st + 8), dict(dx=y + 2), dict(dg=r + 4), dict(db=b + 4), dict(dres=b + 2)):
        assert bwd(**k) == tw.TWEO_ERR_INVALID_ARG, k
    for k in (dict(rows=(1 << 30) + 1), dict(cols=(1 << 24) + 1)):
        assert bwd(**k) == tw.TWEO_ERR_UNSUPPORTED, k
    need = tw.tweo_workspace_bytes(tw.TWEO_OP_LAYERNORM_BWD, 4, 16, 1)
    for k in (dict(ws=None), dict(ws=ws + 8), dict(n=0), dict(n=16)):
        assert bwd(**k) == tw.TWEO_ERR_WORKSPACE, k
    assert need >= 256 and need % 256 == 0
    # the widest rows: partial sums of a few workgroups and not of 512
    assert tw.tweo_workspace_bytes(tw.TWEO_OP_LAYERNORM_BWD, 1 << 20, 1 << 24, 1) <= 4 * (1 << 24) * 4 + (1 << 23) + 256


def entry(memory, **k):
    names = ("param", "master", "grad", "m", "v", "m_step", "v_step")
    t = tw.binding.OptimTensor(*memory[:7], 1000, 0.1, 0, 0)
    t.master = t.m_step = t.v_step = None
    for name, v in k.items():
        setattr(t, name, v)
    assert set(k) <= set(names) | {"n", "weight_decay", "param_f32", "grad_f32"}
    return t


def plan_init(lib, rows, table, bytes_=1 << 14, plan=None):
    plan = plan or tw.binding.OptimPlan()
    return lib.tweo_optim_plan_init((tw.binding.OptimTensor * len(rows))(*rows), len(rows), table, bytes_, ctypes.byref(plan), None)


def test_plan_refusals(lib, memory):
    table, m = memory[8], memory
    second = {k: m[9 + i] for i, k in enumerate(("param", "grad", "m", "v"))}
    bad = [dict(grad=None), dict(m=None), dict(v=None), dict(n=0), dict(n=-5), dict(param_f32=2), dict(grad_f32=-1), dict(param=m[0] + 2),
           dict(grad=m[2] + 2), dict(m=m[3] + 4), dict(v=m[4] + 8), dict(master=m[1] + 4), dict(master=m[1], param_f32=1), dict(m_step=m[5]),
           dict(v_step=m[6]), dict(m_step=m[5] + 4, v_step=m[6]), dict(weight_decay=-0.1), dict(weight_decay=float("nan")),
           dict(weight_decay=float("inf")), dict(param=None),
           # buffers that overlap: the same one twice, one inside another, one that ends in another, the table
           dict(m=m[0]), dict(v=m[3]), dict(master=m[0]), dict(grad=m[0]), dict(grad=m[3] + 1024), dict(v=m[3] + 3984), dict(param=m[2] - 1984),
           dict(v=table), dict(grad=table)]
    for k in bad:
        assert plan_init(lib, [entry(m, **k)], table) == tw.TWEO_ERR_INVALID_ARG, k
        assert plan_init(lib, [entry(m, **second), entry(m, **k)], table) == tw.TWEO_ERR_INVALID_ARG, k
    assert plan_init(lib, [entry(m), entry(m)], table) == tw.TWEO_ERR_INVALID_ARG           # the same tensor twice
    assert plan_init(lib, [entry(m), entry(m, **second, m_step=m[13], v_step=m[14])], table) == tw.TWEO_ERR_INVALID_ARG  # mixed states
    nothing = dict(param=None, m=None, v=None)
    assert plan_init(lib, [entry(m), entry(m, **{**nothing, "grad": m[10]})], table) == tw.TWEO_ERR_INVALID_ARG
    assert plan_init(lib, [entry(m, **{**nothing, "m_step": m[5]})], table) == tw.TWEO_ERR_INVALID_ARG
    assert plan_init(lib, [entry(m, n=(1 << 40) + 1)], table) == tw.TWEO_ERR_UNSUPPORTED
    assert plan_init(lib, [entry(m)], None) == tw.TWEO_ERR_WORKSPACE
    assert plan_init(lib, [entry(m)], table, 64) == tw.TWEO_ERR_WORKSPACE
    assert plan_init(lib, [entry(m)], table + 8) == tw.TWEO_ERR_INVALID_ARG
    rows = (tw.binding.OptimTensor * 1)(entry(m))
    plan = tw.binding.OptimPlan()
    for args in ((None, 1, table, 4096, ctypes.byref(plan)), (rows, 0, table, 4096, ctypes.byref(plan)), (rows, -1, table, 4096, ctypes.byref(plan)),
                 (rows, 1, table, 4096, None)):
        assert lib.tweo_optim_plan_init(*args, None) == tw.TWEO_ERR_INVALID_ARG
    assert lib.tweo_optim_plan_init(rows, (1 << 16) + 1, table, 1 << 30, ctypes.byref(plan), None) == tw.TWEO_ERR_UNSUPPORTED
    assert tw.tweo_optim_table_bytes(0) == 256 and tw.tweo_optim_table_bytes(-3) == 256 and tw.tweo_optim_table_bytes(100) >= 8000


def test_step_refusals(lib, memory):
    t, s, ws = memory[:3]
    plan = tw.binding.OptimPlan(t, 4, 1, 32)
    norm_only, empty = tw.binding.OptimPlan(t, 4, 1, 0), tw.binding.OptimPlan()
    P = ctypes.byref
    need = tw.tweo_workspace_bytes(tw.TWEO_OP_GRAD_SUMSQ, 1, 1, 1)
    for args in ((None, s, ws, need), (P(empty), s, ws, need), (P(plan), None, ws, need), (P(plan), s + 4, ws, need)):
        assert lib.tweo_grad_sumsq(*args, None) == tw.TWEO_ERR_INVALID_ARG
    for args in ((P(plan), s, None, need), (P(plan), s, ws, need - 1), (P(plan), s, ws + 8, need)):
        assert lib.tweo_grad_sumsq(*args, None) == tw.TWEO_ERR_WORKSPACE
    good = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, max_norm=1.0, step=1)

    def step(plan=plan, sumsq=None, schedule=None, **k):
        c = {**good, **k}
        cfg = tw.binding.AdamwCfg(c["lr"], c["beta1"], c["beta2"], c["eps"], c["max_norm"], c["step"])
        return lib.tweo_adamw_step(None if plan is None else P(plan), P(cfg), sumsq, schedule, None)

    nan, inf = float("nan"), float("inf")
    for k in (dict(plan=None), dict(plan=empty), dict(plan=norm_only), dict(lr=-1e-3), dict(lr=nan), dict(lr=inf), dict(beta1=1.0), dict(beta1=-0.1),
              dict(beta2=1.0), dict(beta2=nan), dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(step=0), dict(step=-1), dict(step=1 << 32),
              dict(sumsq=s, max_norm=0.0), dict(sumsq=s, max_norm=nan), dict(sumsq=s + 4), dict(schedule=s + 4), dict(schedule=s, beta1=2.0)):
        assert step(**k) == tw.TWEO_ERR_INVALID_ARG, k
    assert lib.tweo_adamw_step(P(plan), None, None, None, None) == tw.TWEO_ERR_INVALID_ARG


def test_binding_refuses_what_does_not_match():
    f = lambda n, d=torch.float32: torch.zeros(n, dtype=d)  # noqa: E731
    ok = dict(grad=f(600), param=f(600, torch.bfloat16), m=f(600), v=f(600))
    tw.optim_tensor(**ok)
    eight = dict(ok, m=f(600, torch.uint8), v=f(600, torch.uint8), m_step=f(3), v_step=f(3))
    tw.optim_tensor(**eight)
    for k in (dict(grad=f(600, torch.float16)), dict(param=f(599, torch.bfloat16)), dict(param=f(600, torch.float64)), dict(m=f(600, torch.uint8)),
              dict(master=f(600, torch.bfloat16)), dict(v=f(1200)[::2]), dict(m_step=f(3))):
        with pytest.raises(ValueError):
            tw.optim_tensor(**{**ok, **k})
    for k in (dict(m_step=f(2)), dict(v=f(600)), dict(v_step=f(3, torch.float64))):
        with pytest.raises(ValueError):
            tw.optim_tensor(**{**eight, **k})


# ------------------------------------------------------------------------------------------------- pins of the oracle
def test_oracle_layernorm_gradients_are_autograd_s():
    rng = np.random.default_rng(0)
    h, dy, dres = (rng.standard_normal((5, 24)) for _ in range(3))
    gamma, beta = rng.standard_normal(24), rng.standard_normal(24)
    t = [torch.tensor(v, requires_grad=True) for v in (h, gamma, beta)]
    y = torch.nn.functional.layer_norm(t[0], (24,), t[1], t[2], eps=1e-5)
    want = torch.autograd.grad((y * torch.tensor(dy)).sum(), t)
    got = training.layernorm_bwd(dy, h, gamma, training.layernorm_stats(h, 1e-5), dres)
    assert np.allclose(got[0], want[0].numpy() + dres, rtol=1e-12, atol=1e-13)
    assert np.allclose(got[1], want[1].numpy(), rtol=1e-12, atol=1e-13) and np.allclose(got[2], want[2].numpy(), rtol=1e-12)


@pytest.mark.parametrize("clip", [False, True])
def test_oracle_adamw_is_torch_s(clip):
    rng = np.random.default_rng(1)
    p, m, v = rng.standard_normal(50), np.zeros(50), np.zeros(50)
    ref = torch.nn.Parameter(torch.tensor(p))
    opt = torch.optim.AdamW([ref], lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    for t in range(1, 8):
        g = rng.standard_normal(50)
        ref.grad = torch.tensor(g)
        factor = 1.0
        if clip:
            torch.nn.utils.clip_grad_norm_([ref], 1.0)
            factor = training.clip_factor((g * g).sum(), 1.0)
        opt.step()
        p, m, v, _, _ = training.adamw(p, g, m, v, t, 1e-2, 0.9, 0.95, 1e-8, 0.1, factor)
        assert np.allclose(p, ref.detach().numpy(), rtol=1e-12, atol=1e-14)


@pytest.mark.parametrize("fmt,kind", [("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)])
def test_oracle_formats(fmt, kind):
    codes = np.array([c for c in range(256) if (c & 0x7F) <= training.FORMATS[fmt]["largest"]], np.uint8)
    assert np.array_equal(training.decode(codes, fmt), torch.from_numpy(codes).view(kind).double().numpy())


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_oracle_rounds_to_a_neighbour_and_right_on_average(fmt):
    rng = np.random.default_rng(2)
    x = np.abs(rng.standard_normal(512)).astype(np.float32) * np.float32(10.0) ** rng.integers(-6, 1, 512).astype(np.float32)
    values = np.unique(np.abs(training.decode(np.arange(training.FORMATS[fmt]["largest"] + 1, dtype=np.uint8), fmt)))
    total, steps = np.zeros(512), 2000
    for t in range(1, steps + 1):
        value, step, _, _ = training.encode(x, t, fmt)
        total += value
        assert np.isin(value, values).all()
    scaled = x.astype(np.float64) / step[np.arange(512) // 256]
    above = values[np.minimum(np.searchsorted(values, scaled, side="right"), values.size - 1)]
    below = values[np.searchsorted(values, scaled * (1 + 1e-6), side="right") - 1]
    assert np.all(np.abs(value - scaled) <= (above - below) + 1e-6 * scaled)
    # of an evenly spread threshold over `steps` steps the mean is off by a few gaps / steps; below the least code a moment is held up
    # (a block's largest is `top` itself: no gap there, and off by the two roundings of its scale and the product, 2^-22 of it)
    off = np.abs(total / steps - scaled)
    assert np.all((off <= (8 / steps + 1e-4) * (above - below) + 2.0 ** -22 * scaled)[scaled >= 2.0 ** -16]), off.max()
