"""The gated feed-forward's entry points at the ends of what they take, on the GPU."""
import numpy as np
import pytest
import torch

import paper_2511_23225_amd as tw
from oracle import block
from gpu_util import DEV

pytestmark = pytest.mark.gpu
PERIOD = 1 << 20


def say(*a):
    print(*a, flush=True)


def u8(*s):
    return torch.empty(s, dtype=torch.uint8, device=DEV)


def b16(*s):
    return torch.empty(s, dtype=torch.bfloat16, device=DEV)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def repeats(whole, part):
    """Whether the rows of `whole` are those of `part` over and over, to the last one."""
    n = part.shape[0]
    return all(torch.equal(whole[at:at + n], part[:min(n, whole.shape[0] - at)]) for at in range(0, whole.shape[0], n))


def test_gradients_of_most_rows():
    """2^30 rows: as many tiles of 128 as 2^32 threads have workgroups.  Rows that repeat have codes that repeat; no product is asked for."""
    M, F, K = 1 << 30, 8, 16
    say("gated bwd of 2^30 rows")
    g = gen(5)
    dh = torch.randn((PERIOD, F), generator=g, device=DEV, dtype=torch.bfloat16)
    gu = torch.randn((PERIOD, 2 * F), generator=g, device=DEV, dtype=torch.bfloat16)
    sc, ws = torch.ones(16, device=DEV), u8(4096)
    saved = tw.make_saved(u8(16, 16), u8(16, 16), u8(16, 16), u8(16, 16), sc)  # (not looked at)
    q, qT = u8(PERIOD, 2 * F), u8(2 * F, PERIOD)
    tw.tweo_fp8_gated_bwd_bf16(dh, gu, saved, K, q, qT, workspace=ws)
    few = sc[6:9].clone()
    wide, wideT = u8(M, 2 * F), u8(2 * F, M)
    tw.tweo_fp8_gated_bwd_bf16(dh.repeat(M // PERIOD, 1), gu.repeat(M // PERIOD, 1), saved, K, wide, wideT, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(few, sc[6:9]) and torch.equal(qT, q.t())
    assert repeats(wide, q)
    for row, part in zip(wideT, qT):
        assert repeats(row, part)


# Rows whose tiles have 2^32 threads and more: one column of 64x64 tiles of 256 threads and of 512 (the second of two launches holds a few rows), two and three columns
@pytest.mark.parametrize("variant,M,F,keep", [(4, 1 << 30, 8, True), (18, (1 << 29) + 77, 8, False), (4, (1 << 29) + 1000, 64, False)])
def test_fp8_forward_of_most_rows(variant, M, F, keep):
    K = 16
    say("fp8 gated fwd of most rows", variant, M, F)
    g = gen(6)
    code = lambda *s: (torch.randn(s, generator=g, device=DEV) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)  # noqa: E731
    xq, wq = code(PERIOD, K), code(2 * F, K)
    sx, sw = torch.full((4,), 1e-2, device=DEV), torch.full((4,), 1e-2, device=DEV)
    h, gu = b16(PERIOD, F), b16(PERIOD, 2 * F) if keep else None
    many, wide, kept = xq.repeat(-(-M // PERIOD), 1)[:M], b16(M, F), b16(M, 2 * F) if keep else None
    tw.tweo_set_gemm_tile(variant)
    try:
        tw.tweo_fp8_gated_fwd(xq, sx, wq, sw, h, gu_bf16=gu)
        tw.tweo_fp8_gated_fwd(many, sx, wq, sw, wide, gu_bf16=kept)
    finally:
        tw.tweo_set_gemm_tile(0)
    torch.cuda.synchronize()
    bits = lambda t: t.view(torch.int16)  # noqa: E731
    assert repeats(bits(wide), bits(h)) and (not keep or repeats(bits(kept), bits(gu)))
    x, w = (t[:1000].view(torch.float8_e4m3fn).double() for t in (xq, wq))
    p = (x @ w.t() * float(sx[0]) * float(sw[0])).cpu()
    want = torch.nn.functional.silu(p[:, :F]) * p[:, F:]
    # both projections rounded to bf16 (2^-8 each, SiLU's slope to 1.1) after the FP8 products' own error, 2^-10 of the sum of magnitudes; the result once more
    size = (x.abs() @ w.abs().t() * float(sx[0]) * float(sw[0])).cpu()
    off = 2.0 ** -8 * p.abs() + 2.0 ** -9 * size
    bound = 1.1 * off[:, :F] * (p[:, F:].abs() + off[:, F:]) + off[:, F:] * p[:, :F].abs() + 2.0 ** -7 * want.abs() + 1e-30
    assert ((h[:1000].double().cpu() - want).abs() <= bound).all()


@pytest.mark.parametrize("F,i8", [(8, False), (72, True)])
def test_int8_forward_of_most_rows(F, i8):
    M, K = 1 << 30, 16
    say("w8a8 gated of 2^30 rows", F, i8)
    g = gen(7)
    xq, wq = (torch.randint(-127, 128, s, generator=g, device=DEV, dtype=torch.int8) for s in ((PERIOD, K), (2 * F, K)))
    xs, ws = torch.rand(PERIOD, generator=g, device=DEV) * 0.01 + 0.001, torch.rand(2 * F, generator=g, device=DEV) * 0.01 + 0.001
    many, steps = xq.repeat(M // PERIOD, 1), xs.repeat(M // PERIOD)
    few, wide = (torch.empty((n, F), dtype=torch.int8 if i8 else torch.bfloat16, device=DEV) for n in (PERIOD, M))
    for x, s, out in ((xq, xs, few), (many, steps, wide)):
        if i8:
            tw.tweo_w8a8_gated_i8out(x, wq, s, ws, 20.0, out)
        else:
            tw.tweo_w8a8_gated(x, wq, s, ws, out)
    torch.cuda.synchronize()
    assert repeats(wide if i8 else wide.view(torch.int16), few if i8 else few.view(torch.int16))
    p = ((xq[:1000].double() @ wq.double().t()).float() * xs[:1000, None] * ws).double().cpu()
    want = torch.nn.functional.silu(p[:, :F]) * p[:, F:]
    # the sigmoid's argument, its exponential and reciprocal, three products: (|z| + 8) 2^-22 of the value
    got, fp32 = few[:1000].double().cpu(), (p[:, :F].abs() + 8) * 2.0 ** -22 * want.abs()
    if i8:
        assert ((got - (want * 20.0).clamp(-127, 127)).abs() <= 0.5 + 20.0 * fp32).all()
    else:
        assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + fp32 + 2.0 ** -134).all()


@pytest.mark.parametrize("M,K,F", [(1, 272, 136), (70, 144, 40), (130, 1040, 264), (300, 400, 200), (257, 4112, 328)])
def test_int8_forward_on(M, K, F):
    """The kernels that an INT8 call may run on, forced: their sums are exact, so that all give the same bits, and those of fp64 but for the fp32 part."""
    say("w8a8 gated on", M, K, F)
    rng = np.random.default_rng(M + K)
    xq, wq = (torch.from_numpy(rng.integers(-127, 128, s, dtype=np.int8)) for s in ((M, K), (2 * F, K)))
    xs, ws = (torch.from_numpy(rng.uniform(0.5, 2.0, n).astype(np.float32)) * c for n, c in ((M, 1 / 127), (2 * F, 0.03 / K ** 0.5)))
    outs = []
    for variant in (0, 4, 18, 19, 20, 21):
        h, hq = b16(M + 1, F).fill_(7), torch.full((M + 1, F), 7, dtype=torch.int8, device=DEV)
        tw.tweo_set_gemm_tile(variant)
        try:
            tw.tweo_w8a8_gated(xq.to(DEV), wq.to(DEV), xs.to(DEV), ws.to(DEV), h[:M], act="gelu")
            tw.tweo_w8a8_gated_i8out(xq.to(DEV), wq.to(DEV), xs.to(DEV), ws.to(DEV), 30.0, hq[:M], act="gelu")
        finally:
            tw.tweo_set_gemm_tile(0)
        torch.cuda.synchronize()
        assert (h[M:] == 7).all() and (hq[M:] == 7).all()
        outs.append((h.view(torch.int16), hq))
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o, outs[0]))
    p = ((xq.double() @ wq.double().t()).float() * xs[:, None] * ws).double()
    g, u = p[:, :F].numpy(), p[:, F:].numpy()
    want = block.activation(g, "gelu") * u
    z = np.minimum(np.abs(block.gate_argument(g, "gelu")[0]), 130.0)
    fp32 = (z + 8) * 2.0 ** -22 * np.abs(want) + np.where(g < -5, 90 * 2.0 ** -115, 0) * np.abs(u)
    assert (np.abs(outs[0][0][:M].view(torch.bfloat16).double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + fp32 + 2.0 ** -134).all()
    assert (np.abs(outs[0][1][:M].double().cpu().numpy() - np.clip(want * 30.0, -127, 127)) <= 0.5 + 30.0 * (fp32 + 2.0 ** -24 * np.abs(want))).all()
