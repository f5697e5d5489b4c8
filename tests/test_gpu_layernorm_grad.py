"""LayerNorm to bf16 and its gradients through the C ABI, against fp64.

Forward: the kernel normalises in fp64 like the oracle in another summation order, so y is the oracle's bit for bit but where
the fp64 value lies within 1e-10 of a rounding boundary, and the statistics agree to 1e-12.
Backward: fp32, one rounding to bf16 (half a step, 2^-8 of the value).  The fp32 part: with S the sum of the magnitudes of a
result's terms, a sum over a lane's 16 elements, a wave's 6 levels and 8 waves, and the 10 roundings of each term, are within
64 * 2^-24 S.  Column sums: a team's rows one after the other, then a workgroup's teams (8, or 32 where a row has 16 lanes), fp64
then, one rounding to fp32 and 6 roundings in each term; of up to 512 rows 16 one after the other, and the same 7: (rows a team
+ 24) * 2^-24 S, + 40 of up to 128 columns."""
import numpy as np
import pytest
import torch

import oracle
import paper_2511_23225_amd as tw
from oracle import training
from paper_2511_23225_amd import synth
from gpu_util import DEV, to_dev_bf16, bf16_bits, workspace
from test_gpu_layernorm import check_y

pytestmark = pytest.mark.gpu
EPS = 1e-5
GUARD = 64  # elements behind an output that have to stay as they were


def say(*a):
    print(*a, flush=True)


def guarded(shape, dtype, fill):
    n = int(np.prod(shape))
    whole = torch.full((n + GUARD,), fill, dtype=dtype, device=DEV)
    return whole[:n].view(shape), whole[n:]


def untouched(guard, fill):
    return bool((guard == fill).all())


def f64(bits):
    return synth.bf16_bits_to_f32(bits).astype(np.float64)


def inputs(rows, cols, seed):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((rows, cols)) * 2.0 + 0.5).astype(np.float32)
    k = max(1, rows * cols // 5000)
    x.reshape(-1)[rng.choice(rows * cols, k, replace=False)] = rng.uniform(1000, 5000, k)
    b = synth.f32_to_bf16_bits
    n = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    return dict(x=b(x), r=b(n(rows, cols)), gamma=b(1 + 0.1 * n(cols)), beta=b(0.1 * n(cols)), dy=b(n(rows, cols)), dres=b(n(rows, cols)))


# one token; widths on both sides of every change of the waves a row and the pieces a lane has; odd ones; the re-read paths
SHAPES = [(1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (1, 2048), (17, 64), (9, 255), (33, 512), (31, 513), (65, 768), (257, 1001), (12, 1024),
          (13, 1025), (40, 1536), (7, 2048), (6, 2049), (11, 4096), (5, 4104), (3, 8192), (4, 8193), (2, 8200), (3, 16384), (2, 16392), (2, 16385),
          (3, 32776), (2, 33001), (5000, 24), (4099, 768), (3, 253), (3, 257),
          (3, 509), (3, 767), (3, 769), (3, 1023), (3, 1531), (3, 1537), (3, 2047), (3, 4095), (3, 8191), (2, 16383), (300, 8200), (700, 5632),
          (1500, 64), (3001, 61), (1500, 128), (1403, 100), (700, 65), (2001, 129), (999, 256), (1301, 200), (600, 8), (601, 5), (777, 16), (515, 1),
          (512, 768), (513, 768), (512, 1001), (511, 8192), (512, 250), (65, 61)]


def forward(t, cols, residual, beta, stats=True, eps=EPS):
    rows = t["x"].shape[0]
    y, gy = guarded((rows, cols), torch.bfloat16, 7.0)
    h, gh = guarded((rows, cols), torch.bfloat16, 7.0) if residual else (None, None)
    st, gs = guarded((rows, 2), torch.float64, 7.0) if stats else (None, None)
    tw.tweo_layernorm_fwd(to_dev_bf16(t["x"]), to_dev_bf16(t["gamma"]), y, beta_bf16=to_dev_bf16(t["beta"]) if beta else None,
                          residual_bf16=to_dev_bf16(t["r"]) if residual else None, eps=eps, h_out_bf16=h, stats_out=st)
    torch.cuda.synchronize()
    for g in (gy, gh, gs):
        assert g is None or untouched(g, 7.0)
    return y, h, st


@pytest.mark.parametrize("residual,beta", [(False, True), (True, False)])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, residual, beta):
    rows, cols = shape
    say("layernorm fwd", shape, residual)
    t = inputs(rows, cols, rows * 7 + cols)
    y, h, st = forward(t, cols, residual, beta)
    hb = oracle.residual_add_bf16(t["x"], t["r"]) if residual else t["x"]
    if residual:
        assert np.array_equal(bf16_bits(h), hb)
    y64, yb = oracle.layernorm(hb, t["gamma"], t["beta"] if beta else None, float(np.float32(EPS)))
    check_y(bf16_bits(y), yb, y64, shape)
    want = training.layernorm_stats(f64(hb), float(np.float32(EPS)))
    assert np.allclose(st.cpu().numpy(), want, rtol=1e-12, atol=1e-13)
    again, _, _ = forward(t, cols, residual, beta, stats=False)
    assert torch.equal(y, again)


@pytest.mark.parametrize("cols", [3, 48, 100, 256, 777, 768, 1000, 2048, 16392, 33001])
def test_rows_of_one_value(cols):
    """Variance 0: every difference is a zero, whatever 1 / cols rounds to, and y is beta, or a zero whose sign the gain decides."""
    values = np.float32([5.5, -0.1, 3e38, 1e-39, 1 / 3, 0.0, 7.0, -1e30])
    t = inputs(len(values), cols, 3)
    t["x"] = synth.f32_to_bf16_bits(np.repeat(values[:, None], cols, 1))
    t["gamma"][::3] ^= 0x8000
    for beta in (True, False):
        y, _, st = forward(t, cols, False, beta)
        _, yb = oracle.layernorm(t["x"], t["gamma"], t["beta"] if beta else None, float(np.float32(EPS)))
        assert np.array_equal(bf16_bits(y), yb)
        assert np.array_equal(st.cpu().numpy()[:, 0], f64(t["x"])[:, 0])


@pytest.mark.parametrize("eps", [0.0, 1e-30, 0.5, 1e30, float("inf")])
def test_every_eps(eps):
    t = inputs(6, 300, 8)
    y, _, st = forward(t, 300, False, True, eps=eps)
    with np.errstate(all="ignore"):
        want = training.layernorm_stats(f64(t["x"]), float(np.float32(eps)))
    y64, yb = oracle.layernorm(t["x"], t["gamma"], t["beta"], float(np.float32(eps)))
    check_y(bf16_bits(y), yb, y64, eps)
    assert np.allclose(st.cpu().numpy(), want, rtol=1e-12, atol=0)


@pytest.mark.parametrize("shape", [(64, 768), (32, 4096)])
def test_forward_equals_what_the_cast_stores(shape):
    rows, cols = shape
    t = inputs(rows, cols, 5)
    y, h, st = forward(t, cols, True, True)
    y2, h2 = torch.empty_like(y), torch.empty_like(h)
    q = torch.empty(shape, dtype=torch.uint8, device=DEV)
    ws = workspace(tw.TWEO_OP_LAYERNORM_QUANTIZE, rows, 1, 1)
    tw.tweo_layernorm_quantize_e4m3(to_dev_bf16(t["x"]), to_dev_bf16(t["gamma"]), q, ws, beta_bf16=to_dev_bf16(t["beta"]),
                                    residual_bf16=to_dev_bf16(t["r"]), eps=EPS, h_out_bf16=h2, y_out_bf16=y2)
    assert torch.equal(y, y2) and torch.equal(h, h2)
    assert torch.allclose(st, tw.layernorm_stats(ws, rows), rtol=1e-12, atol=1e-13)


def backward(t, h, stats, residual=True, beta=True, dx=None):
    rows, cols = t["dy"].shape
    guard = None
    if dx is None:
        dx, guard = guarded((rows, cols), torch.bfloat16, 7.0)
    dgamma, gg = guarded((cols,), torch.float32, 7.0)
    dbeta, gb = guarded((cols,), torch.float32, 7.0) if beta else (None, None)
    need = tw.tweo_workspace_bytes(tw.TWEO_OP_LAYERNORM_BWD, rows, cols, 1)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV)  # NaNs
    tw.tweo_layernorm_bwd(to_dev_bf16(t["dy"]), h, to_dev_bf16(t["gamma"]), stats, dx, dgamma, dbeta=dbeta,
                          residual_grad_bf16=to_dev_bf16(t["dres"]) if residual else None, workspace=ws[:need])
    torch.cuda.synchronize()
    for g in (guard, gg, gb):
        assert g is None or untouched(g, 7.0)
    assert bool((ws[need:] == 0xFF).all())
    return dx, dgamma, dbeta


def check_backward(t, hb, stats, got, residual=True, beta=True, rows_ok=slice(None)):
    rows = t["dy"].shape[0]
    dx, dgamma, dbeta, size, sg, sb = training.layernorm_bwd(f64(t["dy"]), f64(hb), f64(t["gamma"]), stats, f64(t["dres"]) if residual else None)
    far = np.abs(f64(bf16_bits(got[0])) - dx)
    assert np.all((far <= 2.0 ** -8 * np.abs(dx) + 64 * 2.0 ** -24 * size)[rows_ok]), np.nanmax(far / (size + 1e-300))
    # 512 workgroups of one team of eight waves, 256 of sixteen; of narrow rows 512 workgroups of 32 teams
    cols = t["dy"].shape[1]
    chain = (-(-rows // 16384) + 40 if cols <= 128 else -(-rows // (512 if cols <= 4096 else 256)) + 24) * 2.0 ** -24
    for name, g, ref, s in (("dgamma", got[1], dgamma, sg),) + ((("dbeta", got[2], dbeta, sb),) if beta else ()):
        far = np.abs(g.cpu().numpy().astype(np.float64) - ref)
        assert np.all(far <= chain * s + 1e-30), (name, (far / (s + 1e-300)).max(), chain)


@pytest.mark.parametrize("residual,beta", [(False, True), (True, True), (True, False)])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, residual, beta):
    rows, cols = shape
    say("layernorm bwd", shape, residual, beta)
    t = inputs(rows, cols, rows * 3 + cols)
    stats = training.layernorm_stats(f64(t["x"]), EPS)
    got = backward(t, to_dev_bf16(t["x"]), torch.from_numpy(stats).to(DEV), residual, beta)
    check_backward(t, t["x"], stats, got, residual, beta)
    again = backward(t, to_dev_bf16(t["x"]), torch.from_numpy(stats).to(DEV), residual, beta)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def test_backward_of_the_norm_in_front_of_a_cast():
    """The statistics that the LayerNorm -> cast calls leave in their workspace are what the backward pass takes."""
    rows, cols = 320, 2048
    t = inputs(rows, cols, 23)
    x, r, gamma, beta = (to_dev_bf16(t[k]) for k in ("x", "r", "gamma", "beta"))
    ws = workspace(tw.TWEO_OP_LAYERNORM_QUANTIZE, rows, 1, 1)
    q, h = torch.empty((rows, cols), dtype=torch.uint8, device=DEV), torch.empty_like(x)
    state = torch.zeros(tw.DELAYED_STATE_WORDS, dtype=torch.float32, device=DEV)
    tw.tweo_delayed_state_init(state)
    hb = oracle.residual_add_bf16(t["x"], t["r"])
    stats = training.layernorm_stats(f64(hb), float(np.float32(EPS)))
    for delayed in (False, True):
        ws.fill_(0)
        if delayed:
            tw.tweo_layernorm_quantize_e4m3_delayed(x, gamma, state, q, ws, bootstrap=True, beta_bf16=beta, residual_bf16=r, eps=EPS, h_out_bf16=h)
        else:
            tw.tweo_layernorm_quantize_e4m3(x, gamma, q, ws, beta_bf16=beta, residual_bf16=r, eps=EPS, h_out_bf16=h)
        check_backward(t, hb, stats, backward(t, h, tw.layernorm_stats(ws, rows)))


@pytest.mark.parametrize("shape", [(17501, 768), (3301, 4096), (52000, 256), (1601, 8200), (230001, 64), (110003, 128)])
def test_streams_beyond_the_caches(shape):
    """Calls of more than 100 MB, which read and store past the caches; the second in place."""
    rows, cols = shape
    say("layernorm large", shape)
    t = inputs(rows, cols, rows)
    y, h, st = forward(t, cols, True, True)
    hb = oracle.residual_add_bf16(t["x"], t["r"])
    assert np.array_equal(bf16_bits(h), hb)
    y64, yb = oracle.layernorm(hb, t["gamma"], t["beta"], float(np.float32(EPS)))
    check_y(bf16_bits(y), yb, y64, shape)
    stats = training.layernorm_stats(f64(hb), float(np.float32(EPS)))
    assert np.allclose(st.cpu().numpy(), stats, rtol=1e-12, atol=1e-13)
    got = backward(t, h, st)
    check_backward(t, hb, st.cpu().numpy(), got)
    x, dy = to_dev_bf16(t["x"]), to_dev_bf16(t["dy"])
    y2, dgamma, dbeta = torch.empty_like(x), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    tw.tweo_layernorm_fwd(x, to_dev_bf16(t["gamma"]), y2, beta_bf16=to_dev_bf16(t["beta"]), residual_bf16=to_dev_bf16(t["r"]), eps=EPS, h_out_bf16=x)
    tw.tweo_layernorm_bwd(dy, x, to_dev_bf16(t["gamma"]), st, dy, dgamma, dbeta=dbeta, residual_grad_bf16=to_dev_bf16(t["dres"]),
                          workspace=workspace(tw.TWEO_OP_LAYERNORM_BWD, rows, cols, 1))
    assert torch.equal(x, h) and torch.equal(y2, y) and torch.equal(dy, got[0]) and torch.equal(dgamma, got[1]) and torch.equal(dbeta, got[2])


def test_backward_against_differences():
    """The gradients against central differences of the forward formula in fp64."""
    rows, cols = 3, 40
    t = inputs(rows, cols, 11)
    t["x"] = synth.f32_to_bf16_bits(np.random.default_rng(0).standard_normal((rows, cols)).astype(np.float32))
    x, gamma, dy = f64(t["x"]), f64(t["gamma"]), f64(t["dy"])
    stats = training.layernorm_stats(x, EPS)
    dx, dgamma, dbeta = backward(t, to_dev_bf16(t["x"]), torch.from_numpy(stats).to(DEV), residual=False)

    def loss(x, gamma, beta):
        s = training.layernorm_stats(x, EPS)
        return ((((x - s[:, :1]) * s[:, 1:]) * gamma + beta) * dy).sum()

    step, beta = 1e-5, f64(t["beta"])

    def slope(which, i):
        a = [x.copy(), gamma.copy(), beta.copy()]
        b = [x.copy(), gamma.copy(), beta.copy()]
        a[which].reshape(-1)[i] += step
        b[which].reshape(-1)[i] -= step
        return (loss(*a) - loss(*b)) / (2 * step)

    # the differences: third derivatives of order 10 times step^2, and fp64's 1e-16 * 100 / step
    for which, got, half in ((0, f64(bf16_bits(dx)).reshape(-1), 2.0 ** -8), (1, dgamma.cpu().numpy().astype(np.float64), 2.0 ** -22),
                             (2, dbeta.cpu().numpy().astype(np.float64), 2.0 ** -22)):
        want = np.array([slope(which, i) for i in range(got.size)])
        assert np.all(np.abs(got - want) <= half * np.abs(want) + 1e-5), which


def test_rows_whose_mean_is_far_above_their_deviation():
    rows, cols = 8, 768
    t = inputs(rows, cols, 2)
    rng = np.random.default_rng(3)
    x = (1000.0 + 4.0 * rng.integers(0, 2, (rows, cols))).astype(np.float32)  # neighbouring bf16 values
    x[0] = 5.5                                                                 # and constant rows
    x[1] = 0.0
    t["x"] = synth.f32_to_bf16_bits(x)
    _, _, st = forward(t, cols, False, True)
    stats = training.layernorm_stats(f64(t["x"]), float(np.float32(EPS)))
    assert np.allclose(st.cpu().numpy(), stats, rtol=1e-12, atol=1e-13)
    check_backward(t, t["x"], st.cpu().numpy(), backward(t, to_dev_bf16(t["x"]), st))


@pytest.mark.parametrize("cols", [64, 100, 200, 768, 1001, 4096, 16392])
def test_poisoned_rows_stay_by_themselves(cols):
    rows = 24
    t = inputs(rows, cols, 4)
    clean = forward(t, cols, True, True)
    good = backward(t, clean[1], clean[2])
    x = synth.bf16_bits_to_f32(t["x"]).copy()
    x[3, cols - 1], x[7, 0], x[23, cols // 2] = np.nan, np.inf, -np.inf
    t["x"] = synth.f32_to_bf16_bits(np.nan_to_num(x, nan=0, posinf=0, neginf=0))
    t["x"][3, cols - 1], t["x"][7, 0], t["x"][23, cols // 2] = 0x7FC0, 0x7F80, 0xFF80
    bad = [3, 7, 23]
    rest = [r for r in range(rows) if r not in bad]
    y, h, st = forward(t, cols, True, True)
    assert torch.equal(y[rest], clean[0][rest]) and bool(torch.isnan(y[bad].float()).all())
    dx, dgamma, dbeta = backward(t, h, st)
    assert torch.equal(dx[rest], good[0][rest]) and bool(torch.isnan(dx[bad].float()).all())
    # every column's gain gradient has a NaN term, no bias gradient has
    assert bool(torch.isnan(dgamma).all()) and torch.equal(dbeta, good[2])


@pytest.mark.parametrize("cols", [3, 64, 61, 128, 250, 300, 768, 777, 1001, 2048, 4100, 8192, 16392])
def test_gradients_that_are_not_finite(cols):
    """Infinities and NaNs wherever they lie in a row: what fp64 arithmetic makes of them, in the same places, and the other rows' bits."""
    rows = 9
    t = inputs(rows, cols, 14)
    stats = training.layernorm_stats(f64(t["x"]), EPS)
    clean = backward(t, to_dev_bf16(t["x"]), torch.from_numpy(stats).to(DEV))
    for r, (c, bits) in enumerate(((0, 0x7F80), (cols - 1, 0x7F80), (cols // 2, 0xFF80), (cols - 1, 0xFF80), (cols - 1, 0x7FC0), (0, 0x7FC0))):
        t["dy"][r, c] = bits
    t["dres"][6, cols - 1] = 0x7F80
    got = backward(t, to_dev_bf16(t["x"]), torch.from_numpy(stats).to(DEV))
    with np.errstate(all="ignore"):
        want = training.layernorm_bwd(f64(t["dy"]), f64(t["x"]), f64(t["gamma"]), stats, f64(t["dres"]))
    for g, ref in ((f64(bf16_bits(got[0])), want[0]), (got[1].cpu().numpy(), want[1]), (got[2].cpu().numpy(), want[2])):
        assert np.array_equal(np.isnan(g), np.isnan(ref)) and np.array_equal(g[np.isinf(ref)], ref[np.isinf(ref)]) and np.array_equal(np.isinf(g), np.isinf(ref))
    assert torch.equal(got[0][7:], clean[0][7:]) and torch.equal(got[0][6, :-1], clean[0][6, :-1])


@pytest.mark.parametrize("shape", [(37, 768), (5, 4096), (6, 1001), (3, 33000), (512, 768), (700, 768), (300, 1001), (701, 64), (603, 121)])
def test_in_place(shape):
    rows, cols = shape
    t = inputs(rows, cols, 9)
    y, h, st = forward(t, cols, True, True)
    gamma, beta = to_dev_bf16(t["gamma"]), to_dev_bf16(t["beta"])
    x, r = to_dev_bf16(t["x"]), to_dev_bf16(t["r"])
    tw.tweo_layernorm_fwd(x, gamma, r, beta_bf16=beta, residual_bf16=r, eps=EPS, h_out_bf16=x)  # h in x's place, y in the residual's
    assert torch.equal(x, h) and torch.equal(r, y)
    a = h.clone()
    tw.tweo_layernorm_fwd(a, gamma, a, beta_bf16=beta, eps=EPS)
    assert torch.equal(a, y)
    want = backward(t, h, st)
    for name in ("dy", "dres"):
        dy, dres = to_dev_bf16(t["dy"]), to_dev_bf16(t["dres"])
        dx = dy if name == "dy" else dres
        dgamma, dbeta = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
        tw.tweo_layernorm_bwd(dy, h, gamma, st, dx, dgamma, dbeta=dbeta, residual_grad_bf16=dres,
                              workspace=workspace(tw.TWEO_OP_LAYERNORM_BWD, rows, cols, 1))
        assert torch.equal(dx, want[0]) and torch.equal(dgamma, want[1]) and torch.equal(dbeta, want[2]), name


def test_another_stream_and_a_replayed_graph():
    rows, cols = 200, 768
    t = inputs(rows, cols, 21)
    t2 = inputs(rows, cols, 22)
    x, r, dy = (to_dev_bf16(t[k]) for k in ("x", "r", "dy"))
    gamma, beta = to_dev_bf16(t["gamma"]), to_dev_bf16(t["beta"])
    h, y, dx = (torch.empty_like(x) for _ in range(3))
    st = torch.empty((rows, 2), dtype=torch.float64, device=DEV)
    dgamma, dbeta = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    ws = workspace(tw.TWEO_OP_LAYERNORM_BWD, rows, cols, 1)

    def step():
        tw.tweo_layernorm_fwd(x, gamma, y, beta_bf16=beta, residual_bf16=r, eps=EPS, h_out_bf16=h, stats_out=st)
        tw.tweo_layernorm_bwd(dy, h, gamma, st, dx, dgamma, dbeta=dbeta, residual_grad_bf16=dy, workspace=ws)

    def results():
        torch.cuda.synchronize()
        return [v.clone() for v in (h, y, st, dx, dgamma, dbeta)]

    step()
    want = [results()]
    x.copy_(to_dev_bf16(t2["x"]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    want.append(results())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (0, 1, 0, 1):
        x.copy_(to_dev_bf16((t, t2)[i]["x"]))
        for v in (y, dx, dgamma, ws):
            v.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(results(), want[i])), i
        step()
        assert all(torch.equal(a, b) for a, b in zip(results(), want[i])), i


def test_two_graphs_that_share_a_workspace():
    """Replayed in turn, each leaves what its own eager call does: nothing is kept in the workspace between calls."""
    ws = workspace(tw.TWEO_OP_LAYERNORM_BWD, 3000, 1024, 1)
    cases = []
    for rows, cols in ((3000, 1024), (70, 333)):
        t = inputs(rows, cols, rows)
        stats = torch.from_numpy(training.layernorm_stats(f64(t["x"]), EPS)).to(DEV)
        bufs = [to_dev_bf16(t[k]) for k in ("dy", "x", "gamma", "dres")]
        out = torch.empty_like(bufs[0]), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
        assert ws.nbytes >= tw.tweo_workspace_bytes(tw.TWEO_OP_LAYERNORM_BWD, rows, cols, 1)

        def call(bufs=bufs, out=out, stats=stats):
            tw.tweo_layernorm_bwd(bufs[0], bufs[1], bufs[2], stats, out[0], out[1], dbeta=out[2], residual_grad_bf16=bufs[3], workspace=ws)

        call()
        torch.cuda.synchronize()
        want = [o.clone() for o in out]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        cases.append((graph, out, want, call))
    for i in (0, 1, 1, 0, 0, 1):
        graph, out, want, call = cases[i]
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(out, want)), i


def test_offsets_beyond_32_bits():
    rows, cols = (1 << 16) + 40, 1 << 15  # 2^31 elements and more: byte offsets pass 2^32
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device=DEV)
    t = inputs(40, cols, 1)
    x[-40:] = to_dev_bf16(t["x"])
    x[:-40] = x[-40:-39]
    gamma, beta = to_dev_bf16(t["gamma"]), to_dev_bf16(t["beta"])
    y = torch.empty_like(x)
    st = torch.empty((rows, 2), dtype=torch.float64, device=DEV)
    tw.tweo_layernorm_fwd(x, gamma, y, beta_bf16=beta, eps=EPS, stats_out=st)
    short, st40 = torch.empty((40, cols), dtype=torch.bfloat16, device=DEV), torch.empty((40, 2), dtype=torch.float64, device=DEV)
    tw.tweo_layernorm_fwd(x[-40:], gamma, short, beta_bf16=beta, eps=EPS, stats_out=st40)
    assert torch.equal(y[-40:], short) and torch.equal(st[-40:], st40) and torch.equal(y[0], short[0])
    dgamma, dbeta = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    want = torch.empty_like(short)
    tw.tweo_layernorm_bwd(short, x[-40:], gamma, st40, want, dgamma, dbeta=dbeta, workspace=workspace(tw.TWEO_OP_LAYERNORM_BWD, 40, cols, 1))
    tw.tweo_layernorm_bwd(y, x, gamma, st, y, dgamma, dbeta=dbeta, workspace=workspace(tw.TWEO_OP_LAYERNORM_BWD, rows, cols, 1))
    assert torch.equal(y[-40:], want) and torch.equal(y[0], want[0])


def test_refusals_of_the_binding():
    x = torch.zeros((4, 16), dtype=torch.bfloat16, device=DEV)
    g, y = x[0].clone(), x.clone()
    fwd = tw.tweo_layernorm_fwd
    for bad in (dict(x_bf16=x.float()), dict(y_bf16=y[:2]), dict(y_bf16=torch.zeros((4, 32), dtype=torch.bfloat16, device=DEV)[:, ::2]),
                dict(gamma_bf16=g[:8]), dict(x_bf16=x.cpu()), dict(stats_out=torch.zeros((4, 2), device=DEV)), dict(x_bf16=x[0])):
        with pytest.raises(ValueError):
            fwd(**{**dict(x_bf16=x, gamma_bf16=g, y_bf16=y), **bad})
    with pytest.raises(tw.TweoError):
        fwd(x, g, y, residual_bf16=x)  # nowhere to put h
    with pytest.raises(tw.TweoError):
        fwd(x, g, y, residual_bf16=x, h_out_bf16=y)
    st, d = torch.zeros((4, 2), dtype=torch.float64, device=DEV), torch.zeros(16, device=DEV)
    with pytest.raises(tw.TweoError) as e:
        tw.tweo_layernorm_bwd(x, x, g, st, y, d)
    assert e.value.status == tw.TWEO_ERR_WORKSPACE
    with pytest.raises(ValueError):
        tw.tweo_layernorm_bwd(x, x, g, st.float(), y, d)
    with pytest.raises(ValueError):
        tw.tweo_layernorm_bwd(x, x, g, st, y, d.bfloat16())
