"""The gated feed-forward's entry points through the C ABI, against fp64.

FP8 forward: both projections are held to the bound of the FP8 products (gpu_util.check_gemm: 2^-8 |ref| + (2^-10 + K 2^-24) sum |x w|), the product to what
fp64 makes of the projections as stored: half a bf16 step, and the sigmoid's argument z off by 2 steps (|z| 2^-23 of its value), the
exponential's, the reciprocal's and three products' roundings: (|z| + 8) 2^-22 of the value.  Where the sigmoid is below 2^-115: 90 * 2^-115 |u| absolute.
INT8: the products are exact, so g and u are numpy's fp32 bits.
Gradients: du as the product.  dg = dh u (p + g p (1 - p) z'): p to (|z| + 8) 2^-22 of itself, 1 - p besides to 2^-22 absolute (nothing beyond z = 20,
where fp32's p is 1), the rest 8 roundings.  The codes half a step of their format (2^-4, 2^-3) more, or half the least subnormal."""
import numpy as np
import pytest
import torch

import paper_2511_23225_amd as tw
from oracle import block, training
from gpu_util import DEV

pytestmark = pytest.mark.gpu
GUARD = 64


def say(*a):
    print(*a, flush=True)


def f64(t):
    return t.detach().cpu().double().numpy()


def bf(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16)


def guarded(shape, dtype):
    n = int(np.prod(shape))
    whole = torch.full((n + GUARD,), 7, dtype=dtype, device=DEV)
    return whole[:n].view(shape), whole[n:]


def fp8_gemm_bound(ref, size, K):
    return 2.0 ** -8 * np.abs(ref) + (2.0 ** -10 + K * 2.0 ** -24) * size + 1e-30


def relative(z):
    return (np.minimum(np.abs(z), 130.0) + 8) * 2.0 ** -22


def product_bound(g, u, act):
    """Of the fp32 part of act(g) * u."""
    z, _ = block.gate_argument(g, act)
    return relative(z) * np.abs(block.activation(g, act) * u) + np.where(z < -79, 90 * 2.0 ** -115, 0) * np.abs(u) + 2.0 ** -134


def codes(shape, rng, top=448.0, fmt=torch.float8_e4m3fn):
    x = torch.from_numpy(rng.standard_normal(shape).astype(np.float32))
    x.view(-1)[rng.integers(0, x.numel(), 1 + x.numel() // 3000)] *= 20.0
    s = top / float(x.abs().max())
    return (x * s).to(fmt).view(torch.uint8), s


# one row to several tiles; columns and contractions that end inside tiles, stages and 16-byte chunks
FP8_SHAPES = [(1, 8, 16), (1, 256, 128), (2, 24, 48), (5, 1000, 528), (17, 40, 144), (64, 32, 256), (65, 64, 384), (100, 136, 2048), (130, 72, 272),
              (300, 1000, 528), (257, 512, 1040), (1, 5632, 2048), (33, 4096, 512), (512, 2048, 768), (700, 1336, 112), (1023, 3000, 640), (2049, 264, 1296)]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("shape", FP8_SHAPES)
def test_fp8_forward(shape, act):
    M, F, K = shape
    say("fp8 gated fwd", shape, act)
    check_fp8_forward(M, F, K, act)


def check_fp8_forward(M, F, K, act, rows=None, seed=0):
    rng = np.random.default_rng(M * 7 + F * 3 + K + seed)
    xq, sx = codes((M, K), rng)
    wq, sw = codes((2 * F, K), rng)
    # gates from far below to far above nothing
    sxi, swi = torch.full((4,), 1 / sx, device=DEV), torch.full((4,), 3.0 / np.sqrt(K) / sw, device=DEV)
    h, gh = guarded((M, F), torch.bfloat16)
    gu, gg = guarded((M, 2 * F), torch.bfloat16)
    xd, wd = xq.to(DEV), wq.to(DEV)
    tw.tweo_fp8_gated_fwd(xd, sxi, wd, swi, h, gu_bf16=gu, act=act)
    alone, ga = guarded((M, F), torch.bfloat16)
    tw.tweo_fp8_gated_fwd(xd, sxi, wd, swi, alone, act=act)
    torch.cuda.synchronize()
    assert all((g == 7).all() for g in (gh, gg, ga))
    assert torch.equal(h.view(torch.int16), alone.view(torch.int16))
    pick = np.arange(M) if rows is None else rng.choice(M, rows, replace=False)
    x, w = training.decode(xq.numpy()[pick], "e4m3"), training.decode(wq.numpy(), "e4m3")
    alpha = float(sxi[0]) * float(swi[0])
    ref, size = x @ w.T * alpha, np.abs(x) @ np.abs(w).T * alpha
    got = f64(gu)[pick]
    off = np.abs(got - ref) / fp8_gemm_bound(ref, size, K)
    assert off.max() <= 1, off.max()
    g, u = got[:, :F], got[:, F:]
    want = block.activation(g, act) * u
    off = np.abs(f64(h)[pick] - want) / (2.0 ** -8 * np.abs(want) + product_bound(g, u, act))
    assert off.max() <= 1, off.max()


# the kernels that a call may run on, forced: 64x64 tiles (4, 18), 64x128 (19, 20), 128x128 (21), the deferred-epilogue kernel on whole tiles (15) and
# with edges (24); where a variant does not take the sizes the usual choice runs
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("variant,shape", [(4, (130, 136, 272)), (18, (70, 40, 144)), (18, (65, 1000, 1040)), (19, (130, 136, 272)), (19, (64, 64, 128)), (20, (200, 328, 656)),
                                           (20, (1, 64, 16)), (21, (300, 200, 400)), (21, (128, 64, 1152)),
                                           (15, (256, 128, 768)), (15, (512, 256, 896)), (15, (1024, 2176, 1024)), (15, (768, 384, 1920)), (15, (2304, 4352, 2048)),
                                           (15, (256, 128, 2176)), (24, (192, 128, 1024)), (24, (1, 8, 912)), (24, (193, 136, 928)), (24, (700, 1000, 1296)),
                                           (24, (1000, 8200, 1168)), (24, (3000, 2056, 2320)), (24, (385, 264, 4096)), (24, (2049, 4104, 1024))])
def test_fp8_forward_on(variant, shape, act):
    M, F, K = shape
    say("fp8 gated fwd on", variant, shape, act)
    tw.tweo_set_gemm_tile(variant)
    try:
        check_fp8_forward(M, F, K, act, rows=min(M, 300))
    finally:
        tw.tweo_set_gemm_tile(0)


@pytest.mark.parametrize("variant,M,F,K", [(21, 262200, 8200, 16), (15, 262144, 8192, 768), (24, 262100, 8200, 928)])
def test_fp8_outputs_beyond_32_bits(variant, M, F, K):
    """h of more than 2^32 bytes, both projections of twice as many: the last rows, and some in between, against fp64."""
    say("fp8 gated fwd of many rows", variant, M, F, K)
    g = torch.Generator(device=DEV).manual_seed(3)
    code = lambda *s: (torch.randn(s, generator=g, device=DEV) * 60).clamp(-448, 448).to(torch.float8_e4m3fn)  # noqa: E731
    xq, wq = code(M, K), code(2 * F, K)
    sx, sw = torch.full((4,), 1e-2, device=DEV), torch.full((4,), 0.05 / K ** 0.5, device=DEV)
    h, gh = guarded((M, F), torch.bfloat16)
    gu, gg = guarded((M, 2 * F), torch.bfloat16)
    tw.tweo_set_gemm_tile(variant)
    try:
        tw.tweo_fp8_gated_fwd(xq.view(torch.uint8), sx, wq.view(torch.uint8), sw, h, gu_bf16=gu)
    finally:
        tw.tweo_set_gemm_tile(0)
    torch.cuda.synchronize()
    assert (gh == 7).all() and (gg == 7).all()
    rows = torch.tensor([0, 1, 131071, 131072, 200003, M - 2, M - 1], device=DEV)
    x, w = f64(xq[rows].float()), f64(wq.float())
    alpha = float(sx[0]) * float(sw[0])
    ref, size = x @ w.T * alpha, np.abs(x) @ np.abs(w).T * alpha
    got = f64(gu[rows])
    assert (np.abs(got - ref) <= fp8_gemm_bound(ref, size, K)).all()
    want = block.activation(got[:, :F], "silu") * got[:, F:]
    assert (np.abs(f64(h[rows]) - want) <= 2.0 ** -8 * np.abs(want) + product_bound(got[:, :F], got[:, F:], "silu")).all()


def test_gradients_beyond_32_bits():
    """Codes of more than 2^32 bytes, and their transposed copy: some rows and columns against fp64."""
    M, F, K = 262144, 8200, 16
    say("gated bwd of many rows", M, F)
    g = torch.Generator(device=DEV).manual_seed(4)
    dh, gu = torch.randn((M, F), generator=g, device=DEV, dtype=torch.bfloat16), torch.randn((M, 2 * F), generator=g, device=DEV, dtype=torch.bfloat16)
    t = saved_of(16, 16, K, np.random.default_rng(0))  # (no product is asked for)
    q, gq = guarded((M, 2 * F), torch.uint8)
    qT, gqT = guarded((2 * F, M), torch.uint8)
    ws = torch.empty(4096, dtype=torch.uint8, device=DEV)
    tw.tweo_fp8_gated_bwd_bf16(dh, gu, t["saved"], K, q, qT, workspace=ws)
    torch.cuda.synchronize()
    assert (gq == 7).all() and (gqT == 7).all()
    scale = float(t["sc"][7])
    for rows in (slice(0, 64), slice(131040, 131104), slice(M - 64, M)):
        want, bound = grad_reference(f64(dh[rows]), f64(gu[rows]), "silu")
        got = training.decode(q[rows].cpu().numpy(), "e4m3") / scale
        off = np.abs(got - want) / (np.maximum(2.0 ** -4 * (1 + 2.0 ** -7) * np.abs(want), 2.0 ** -10 / scale) + 2.0 ** -8 * np.abs(want) + 2 * bound)
        assert off.max() <= 1, off.max()
        assert torch.equal(q[rows], qT[:, rows].t())


def test_fp8_special_values():
    """A NaN code spoils its row, or its column and no other; projections that are infinite or overflow give what the formula gives."""
    M, F, K = 70, 72, 144
    rng = np.random.default_rng(5)
    xq, wq = codes((M, K), rng)[0], codes((2 * F, K), rng)[0]
    xq[3, 7], wq[5, 9], wq[F + 11, 0] = 0x7F, 0xFF, 0x7F
    one = torch.ones(4, device=DEV) * 1e-3
    h, gu = torch.empty((M, F), dtype=torch.bfloat16, device=DEV), torch.empty((M, 2 * F), dtype=torch.bfloat16, device=DEV)
    tw.tweo_fp8_gated_fwd(xq.to(DEV), one, wq.to(DEV), one, h, gu_bf16=gu)
    bad = np.zeros((M, F), bool)
    bad[3] = bad[:, 5] = bad[:, 11] = True
    assert (np.isnan(f64(h)) == bad).all()
    for scale in (1e35, 1e12, 1e-30):
        s = torch.full((4,), scale, device=DEV)
        xq[3, 7], wq[5, 9], wq[F + 11, 0] = 0, 0, 0
        for act in ("silu", "gelu"):
            tw.tweo_fp8_gated_fwd(xq.to(DEV), s, wq.to(DEV), torch.ones(4, device=DEV), h, gu_bf16=gu, act=act)
            g, u = f64(gu)[:, :F], f64(gu)[:, F:]
            with np.errstate(invalid="ignore"):
                want = np.where(g > 0, g, 0.0) * u if scale > 1 else 0.5 * g * u  # (a sum of codes is no small number: 448^2 / 2^18 at least, or 0)
                got, fine = f64(h), np.isfinite(g) & (np.abs(want) < 3e38) & ((np.abs(g) > 1e4) | (scale < 1))
                assert (np.abs(got - want) <= 2.0 ** -7 * np.abs(want) + 1e-37)[fine].all()
            assert not np.isnan(got[np.isfinite(g) & np.isfinite(u)]).any()


W8_SHAPES = [(1, 8, 16), (1, 256, 64), (1, 11008, 4096), (3, 1000, 528), (16, 264, 1040), (17, 40, 144), (64, 32, 256), (64, 5632, 2048), (65, 64, 384), (130, 72, 272),
             (300, 1000, 528), (257, 512, 1040), (1000, 1336, 112), (513, 2056, 4096)]


@pytest.mark.parametrize("tokens,channels", [(True, True), (False, False), (True, False), (False, True)])
@pytest.mark.parametrize("shape", W8_SHAPES)
def test_w8a8(shape, tokens, channels):
    M, F, K = shape
    act = "silu" if tokens else "gelu"
    say("w8a8 gated", shape, act, tokens, channels)
    rng = np.random.default_rng(M + F + K)
    xq, wq = rng.integers(-127, 128, (M, K), dtype=np.int8), rng.integers(-127, 128, (2 * F, K), dtype=np.int8)
    xs = (rng.uniform(0.5, 2.0, M if tokens else 1) / 127).astype(np.float32)
    ws = (rng.uniform(0.5, 2.0, 2 * F if channels else 1) * 0.03 / np.sqrt(K)).astype(np.float32)
    dev = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    h, gh = guarded((M, F), torch.bfloat16)
    hq, gq = guarded((M, F), torch.int8)
    args = dev(xq), dev(wq), dev(xs), dev(ws)
    tw.tweo_w8a8_gated(*args, h, act=act)
    inv = 40.0
    tw.tweo_w8a8_gated_i8out(*args, inv, hq, act=act)
    torch.cuda.synchronize()
    assert (gh == 7).all() and (gq == 7).all()
    pick = np.arange(M) if M * F * K < 1 << 28 else rng.choice(M, max(1, (1 << 28) // (F * K)), replace=False)
    acc = xq[pick].astype(np.float64) @ wq.astype(np.float64).T  # whole numbers below 2^53
    gu = (acc.astype(np.float32) * (xs[pick][:, None] if tokens else xs)) * ws
    g, u = gu[:, :F].astype(np.float64), gu[:, F:].astype(np.float64)
    want, bound = block.activation(g, act) * u, product_bound(g, u, act)
    off = np.abs(f64(h)[pick] - want) / (2.0 ** -8 * np.abs(want) + bound)
    assert off.max() <= 1, off.max()
    q = f64(hq)[pick]
    assert (np.abs(q - np.clip(want * inv, -127, 127)) <= 0.5 + inv * (bound + 2.0 ** -24 * np.abs(want))).all()


def test_w8a8_extremes():
    """The largest sums, a step that is not a number, a result beyond the INT8 range."""
    M, F, K = 4, 16, 8192
    x, w = torch.full((M, K), 127, dtype=torch.int8, device=DEV), torch.full((2 * F, K), 127, dtype=torch.int8, device=DEV)
    w[F:] = -127
    h, hq = torch.empty((M, F), dtype=torch.bfloat16, device=DEV), torch.empty((M, F), dtype=torch.int8, device=DEV)
    s = torch.tensor([1.0, float("nan"), 2.0, 1e-6], device=DEV)
    tw.tweo_w8a8_gated(x, w, s, torch.ones(1, device=DEV), h)
    tw.tweo_w8a8_gated_i8out(x, w, s, torch.ones(1, device=DEV), 1.0, hq)
    a = float(127 * 127 * 8192)
    got = f64(h)
    assert (np.abs(got[0] + a * a) <= 2.0 ** -7 * a * a).all() and np.isnan(got[1]).all() and (np.abs(got[2] + 4 * a * a) <= 2.0 ** -7 * 4 * a * a).all()
    assert (f64(hq)[0] == -127).all() and (f64(hq)[1] == 0).all()


# ---- backward
def saved_of(M, N, K, rng):
    """What a forward pass leaves."""
    (xq, sx), (wq, sw) = codes((M, K), rng), codes((N, K), rng)
    u8 = lambda t: t.to(DEV).contiguous()  # noqa: E731
    t = dict(xq=u8(xq), xqT=u8(xq.t()), wq=u8(wq), wqT=u8(wq.t()), sc=torch.zeros(16, device=DEV))
    t["sc"][:6] = torch.tensor([448 / sx, sx, 1 / sx, 448 / sw, sw, 1 / sw])
    t["saved"] = tw.make_saved(t["xq"], t["xqT"], t["wq"], t["wqT"], t["sc"])
    return t


def grad_reference(dh, gu, act):
    F = dh.shape[1]
    g, u = gu[:, :F], gu[:, F:]
    z, dz = block.gate_argument(g, act)
    with np.errstate(over="ignore"):
        p, rest = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z))
    inner = np.where(p * rest == 0, 0, rest * 2 * relative(z) * np.abs(g) * p * dz) + np.where(z < 20, 2.0 ** -22 * np.abs(g) * p * dz, 0)
    bound = np.abs(dh * u) * (2 * relative(z) * p + inner + 8 * 2.0 ** -24 * np.abs(block.activation_slope(g, act)) + np.where(z < -79, 90 * 2.0 ** -110, 0))
    return (np.concatenate([dh * u * block.activation_slope(g, act), dh * block.activation(g, act)], 1),
            np.concatenate([bound + 2.0 ** -134, product_bound(g, dh, act)], 1))


GRAD_SHAPES = [(16, 8, 16), (16, 24, 48), (32, 128, 128), (48, 136, 272), (144, 40, 64), (256, 512, 512), (1024, 200, 128), (400, 1000, 176), (2064, 264, 144)]


@pytest.mark.parametrize("e5m2", [False, True])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("shape", GRAD_SHAPES)
def test_backward(shape, act, e5m2):
    M, F, K = shape
    say("gated bwd", shape, act, e5m2)
    rng = np.random.default_rng(M + F + K)
    t = saved_of(M, 2 * F, K, rng)
    gu = rng.standard_normal((M, 2 * F)) * 3
    gu[rng.integers(0, M, 5), rng.integers(0, 2 * F, 5)] = [50.0, -50.0, 1000.0, -1000.0, 0.0]
    dh, gu = bf(rng.standard_normal((M, F)) * 1e-3), bf(gu)
    q, gq = guarded((M, 2 * F), torch.uint8)
    qT, gqT = guarded((2 * F, M), torch.uint8)
    dx, gx = guarded((M, K), torch.bfloat16)
    dw, gw = guarded((2 * F, K), torch.bfloat16)
    ws = torch.empty(tw.tweo_workspace_bytes(tw.TWEO_OP_FP8_GATED_BWD_BF16, M, F, K), dtype=torch.uint8, device=DEV)
    call = lambda dx, dw: tw.tweo_fp8_gated_bwd_bf16(dh.to(DEV), gu.to(DEV), t["saved"], K, q, qT, dx_bf16=dx, dw_bf16=dw, act=act, dy_e5m2=e5m2, workspace=ws)  # noqa: E731
    call(dx, dw)
    torch.cuda.synchronize()
    assert all((g == 7).all() for g in (gq, gqT, gx, gw))
    fmt, top = ("e5m2", 57344.0) if e5m2 else ("e4m3", 448.0)
    want, bound = grad_reference(f64(dh), f64(gu), act)
    amax, scale, inv = (float(v) for v in t["sc"][6:9].cpu())
    at = np.unravel_index(np.abs(want).argmax(), want.shape)
    assert abs(amax - abs(want[at])) <= 2.0 ** -8 * amax + bound[at]
    assert scale == float(np.float32(top) / np.float32(amax)) and inv == float(np.float32(1) / np.float32(scale))
    assert torch.equal(qT, q.t())
    got = training.decode(q.cpu().numpy(), fmt) / scale
    step = 2.0 ** (-3 if e5m2 else -4)
    least = 2.0 ** (-17 if e5m2 else -10) / scale  # half the least subnormal
    off = np.abs(got - want) / (np.maximum(step * (1 + 2.0 ** -7) * np.abs(want), least) + 2.0 ** -8 * np.abs(want) + 2 * bound)
    assert off.max() <= 1, off.max()
    # the products are those of the linears on these codes
    dx2, dw2 = torch.empty_like(dx), torch.empty_like(dw)
    linear = tw.tweo_fp8_linear_bwd_hybrid if e5m2 else tw.tweo_fp8_linear_bwd
    linear(q, qT, t["sc"][8:9], t["wqT"], t["sc"][5:6], t["xqT"], t["sc"][2:3], M, 2 * F, K, dx2, dw2, ws[4096:])
    assert torch.equal(dx.view(torch.int16), dx2.view(torch.int16)) and torch.equal(dw.view(torch.int16), dw2.view(torch.int16))
    # one of the two, or none
    one, other = torch.full_like(dx, 7), torch.full_like(dw, 7)
    call(one, None)
    call(None, other)
    call(None, None)
    bound = lambda a, b: fp8_gemm_bound(a @ b, np.abs(a) @ np.abs(b), a.shape[1])  # noqa: E731
    for got, a, b in ((one, training.decode(q.cpu().numpy(), fmt) * inv, training.decode(t["wq"].cpu().numpy(), "e4m3") * float(t["sc"][5])),
                      (other, training.decode(qT.cpu().numpy(), fmt) * inv, training.decode(t["xq"].cpu().numpy(), "e4m3") * float(t["sc"][2]))):
        assert (np.abs(f64(got) - a @ b) <= bound(a, b)).all()


def test_backward_delayed():
    """A scale that was fixed before: the history, what a call uses and what it leaves."""
    for e5m2 in (False, True):
        top = 57344.0 if e5m2 else 448.0
        for M, F in ((32, 40), (1024, 1000), (4096, 2048)):
            rng = np.random.default_rng(3)
            t, K = saved_of(M, 2 * F, 16, rng), 16
            state = torch.empty(tw.DELAYED_STATE_WORDS, dtype=torch.float32, device=DEV)
            tw.tweo_delayed_state_init(state)
            ws = torch.empty(tw.tweo_workspace_bytes(tw.TWEO_OP_FP8_GATED_BWD_BF16, M, F, K), dtype=torch.uint8, device=DEV)
            q, qT = (torch.empty(s, dtype=torch.uint8, device=DEV) for s in ((M, 2 * F), (2 * F, M)))
            history, nxt = [], None
            for i in range(4):
                say("gated bwd delayed", e5m2, M, F, i)
                size = [1e-3, 3e-3, 1e-4, 1e-3][i]
                dh, gu = bf(rng.standard_normal((M, F)) * size), bf(rng.standard_normal((M, 2 * F)))
                run = lambda **k: tw.tweo_fp8_gated_bwd_bf16(dh.to(DEV), gu.to(DEV), t["saved"], K, q, qT, dy_e5m2=e5m2, workspace=ws, **k)  # noqa: E731
                run()
                now = t["sc"][6:9].cpu().numpy().copy()
                plain = q.clone()
                run(state_dgu=state, bootstrap=i == 0)
                sc, words = t["sc"][6:9].cpu().numpy(), state.cpu().numpy()
                assert sc[0] == now[0] and words[16] == 0 and (sc[1:3] == words[21:23]).all()
                history.append(sc[0])
                assert sc[1] == (now[1] if i == 0 else nxt)
                nxt = words[17]
                assert nxt == np.float32(top) / np.float32(max(history)) and words[18] == np.float32(1) / nxt
                assert words[:16].tolist() == history + [0.0] * (16 - len(history))
                assert torch.equal(qT, q.t())
                if sc[1] == now[1]:
                    assert torch.equal(q, plain)
                want, bound = grad_reference(f64(dh), f64(gu), "silu")
                want = np.clip(want, -top / sc[1], top / sc[1])
                got = training.decode(q.cpu().numpy(), "e5m2" if e5m2 else "e4m3") / float(sc[1])
                step, least = 2.0 ** (-3 if e5m2 else -4), 2.0 ** (-17 if e5m2 else -10) / float(sc[1])
                assert (np.abs(got - want) <= np.maximum(step * (1 + 2.0 ** -7) * np.abs(want), least) + 2.0 ** -8 * np.abs(want) + 2 * bound).all()


def test_backward_of_zeros_and_infinities():
    M, F, K = 32, 24, 16
    t = saved_of(M, 2 * F, K, np.random.default_rng(1))
    ws = torch.empty(tw.tweo_workspace_bytes(tw.TWEO_OP_FP8_GATED_BWD_BF16, M, F, K), dtype=torch.uint8, device=DEV)
    q, qT = (torch.empty(s, dtype=torch.uint8, device=DEV) for s in ((M, 2 * F), (2 * F, M)))
    gu = torch.randn((M, 2 * F), device=DEV).bfloat16()
    dh = torch.zeros((M, F), dtype=torch.bfloat16, device=DEV)
    run = lambda: tw.tweo_fp8_gated_bwd_bf16(dh, gu, t["saved"], K, q, qT, workspace=ws)  # noqa: E731
    run()
    assert t["sc"][6:9].tolist() == [0.0, 1.0, 1.0] and ((q & 0x7F) == 0).all()
    dh[5, 6] = float("nan")
    run()
    bad = torch.zeros((M, 2 * F), dtype=torch.bool, device=DEV)
    bad[5, 6] = bad[5, F + 6] = True
    assert torch.isnan(t["sc"][6]) and t["sc"][7] == 1 and (((q & 0x7F) == 0x7F) == bad).all()


# ---- from bf16 operands
@pytest.mark.parametrize("shape", [(32, 40, 48), (256, 512, 512), (1024, 1000, 256), (4096, 2048, 1024)])
@pytest.mark.parametrize("delayed", [False, True])
def test_forward_from_bf16(shape, delayed):
    """Codes, scalars and results are those of the linear's entry point for the same weight and of the kernel on its codes."""
    M, F, K = shape
    say("gated fwd bf16", shape, delayed)
    rng = np.random.default_rng(9)
    x, w = bf(rng.standard_normal((M, K))).to(DEV), bf(rng.standard_normal((2 * F, K)) * 0.05).to(DEV)
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device=DEV)  # noqa: E731
    outs, states = [], []
    for linear in (True, False):
        buf = [u8(M, K), u8(K, M), u8(2 * F, K), u8(K, 2 * F)]
        sc = torch.zeros(16, device=DEV)
        saved = tw.make_saved(*buf, sc)
        gu, h = torch.empty((M, 2 * F), dtype=torch.bfloat16, device=DEV), torch.empty((M, F), dtype=torch.bfloat16, device=DEV)
        st = [torch.empty(32, device=DEV) for _ in range(2)]
        [tw.tweo_delayed_state_init(s) for s in st]
        op = tw.TWEO_OP_FP8_LINEAR_FWD_BF16 if linear else tw.TWEO_OP_FP8_GATED_FWD_BF16
        ws = torch.empty(tw.tweo_workspace_bytes(op, M, 2 * F if linear else F, K), dtype=torch.uint8, device=DEV)
        for step in range(2):
            if linear and delayed:
                tw.tweo_fp8_linear_fwd_bf16_delayed(x, w, gu, saved, *st, bootstrap=step == 0, workspace=ws)
            elif linear:
                tw.tweo_fp8_linear_fwd_bf16(x, w, gu, saved, workspace=ws)
            elif delayed:
                tw.tweo_fp8_gated_fwd_bf16(x, w, h, gu, saved, state_x=st[0], state_w=st[1], bootstrap=step == 0)
            else:
                tw.tweo_fp8_gated_fwd_bf16(x, w, h, gu, saved, workspace=ws)
        torch.cuda.synchronize()
        outs.append(buf + [sc[:6].clone()] + st)
        states.append((gu, h, sc, buf))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    (gu, _, _, _), (gu2, h, sc, buf) = states
    assert (gu.float() - gu2.float()).abs().max() <= 2.0 ** -7 * gu.float().abs().max()
    again, kept = torch.empty_like(h), torch.empty_like(gu2)
    tw.tweo_fp8_gated_fwd(buf[0], sc[2:3], buf[2], sc[5:6], again, gu_bf16=kept)
    assert torch.equal(again.view(torch.int16), h.view(torch.int16)) and torch.equal(kept.view(torch.int16), gu2.view(torch.int16))


def test_streams_and_graphs():
    """A forward and backward pass on a stream of its own, and captured: replays with other data, eager calls and a second graph of the same
    buffers (workspaces of their own) in between."""
    M, F, K = 272, 264, 144
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device=DEV)  # noqa: E731
    b16 = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    x, w, dh, h, gu, dx, dw = b16(M, K), b16(2 * F, K), b16(M, F), b16(M, F), b16(M, 2 * F), b16(M, K), b16(2 * F, K)
    buf, sc, q, qT = [u8(M, K), u8(K, M), u8(2 * F, K), u8(K, 2 * F)], torch.zeros(16, device=DEV), u8(M, 2 * F), u8(2 * F, M)
    saved = tw.make_saved(*buf, sc)
    xi, wi = torch.zeros((M, K), dtype=torch.int8, device=DEV), torch.zeros((2 * F, K), dtype=torch.int8, device=DEV)
    xs, wsx, h8 = torch.ones(M, device=DEV) * 0.01, torch.ones(2 * F, device=DEV) * 0.002, b16(M, F)
    ws = [u8(max(tw.tweo_workspace_bytes(op, M, F, K) for op in (tw.TWEO_OP_FP8_GATED_FWD_BF16, tw.TWEO_OP_FP8_GATED_BWD_BF16))) for _ in range(2)]

    def load(seed):
        g = torch.Generator().manual_seed(seed)
        for t, s in ((x, 1.0), (w, 0.05), (dh, 1e-3)):
            t.copy_(torch.randn(t.shape, generator=g) * s)
        for t in (xi, wi):
            t.copy_(torch.randint(-127, 128, t.shape, generator=g))

    def step(ws):
        tw.tweo_fp8_gated_fwd_bf16(x, w, h, gu, saved, workspace=ws)
        tw.tweo_fp8_gated_bwd_bf16(dh, gu, saved, K, q, qT, dx, dw, workspace=ws)
        tw.tweo_w8a8_gated(xi, wi, xs, wsx, h8)

    def result():
        torch.cuda.synchronize()
        return [t.clone().view(torch.int16 if t.dtype is torch.bfloat16 else t.dtype) for t in (h, gu, dx, dw, q, sc[:9], h8)]

    eager = []
    for seed in range(3):
        load(seed)
        step(ws[0])
        eager.append(result())
    side = torch.cuda.Stream()
    load(1)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(ws[1])
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(result(), eager[1]))
    graphs = []
    for s in ws:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(s)
        graphs.append(g)
    for seed in (0, 1, 2, 0, 1):
        for g in graphs:
            load(seed)
            g.replay()
            assert all(torch.equal(a, b) for a, b in zip(result(), eager[seed])), seed
        load(2 - seed)
        step(ws[0])
        assert all(torch.equal(a, b) for a, b in zip(result(), eager[2 - seed]))


def test_binding_refusals():
    M, F, K = 32, 24, 16
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device=DEV)  # noqa: E731
    b16 = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    one, h, gu = torch.ones(4, device=DEV), b16(M, F), b16(M, 2 * F)
    good = dict(xq=u8(M, K), sx_inv=one, wq=u8(2 * F, K), sw_inv=one, h_bf16=h, gu_bf16=gu)
    tw.tweo_fp8_gated_fwd(**good)
    for k in (dict(act="relu"), dict(wq=u8(2 * F + 1, K)), dict(wq=u8(2 * F, 32)), dict(xq=u8(M, 2 * K)[:, ::2]), dict(h_bf16=b16(M, 2 * F)),
              dict(gu_bf16=b16(M, F)), dict(h_bf16=h.float()), dict(sx_inv=one.double()), dict(sx_inv=one.cpu()), dict(xq=u8(M, K).view(torch.int8))):
        with pytest.raises(ValueError):
            tw.tweo_fp8_gated_fwd(**{**good, **k})
    i8 = lambda *s: torch.zeros(s, dtype=torch.int8, device=DEV)  # noqa: E731
    good = dict(xq=i8(M, K), wq=i8(2 * F, K), x_step=one[:1], w_step=one[:1], h_bf16=h)
    tw.tweo_w8a8_gated(**good)
    for k in (dict(x_step=one[:2]), dict(w_step=torch.ones(F, device=DEV)), dict(x_step=one[:1].double()), dict(wq=i8(2 * F, K)[::2]), dict(h_bf16=gu)):
        with pytest.raises(ValueError):
            tw.tweo_w8a8_gated(**{**good, **k})
    t = saved_of(M, 2 * F, K, np.random.default_rng(0))
    ws = u8(tw.tweo_workspace_bytes(tw.TWEO_OP_FP8_GATED_BWD_BF16, M, F, K))
    good = dict(dh_bf16=h, gu_bf16=gu, saved=t["saved"], K=K, dguq=u8(M, 2 * F), dguqT=u8(2 * F, M), dx_bf16=b16(M, K), dw_bf16=b16(2 * F, K), workspace=ws)
    tw.tweo_fp8_gated_bwd_bf16(**good)
    for k in (dict(gu_bf16=b16(M, F)), dict(dguqT=u8(M, 2 * F)), dict(dx_bf16=b16(K, M)), dict(dw_bf16=b16(F, K)), dict(state_dgu=one), dict(act="none"),
              dict(workspace=ws[::2])):
        with pytest.raises(ValueError):
            tw.tweo_fp8_gated_bwd_bf16(**{**good, **k})
    for k in (dict(workspace=None), dict(workspace=ws[:4080])):
        with pytest.raises(tw.TweoError):
            tw.tweo_fp8_gated_bwd_bf16(**{**good, **k})
