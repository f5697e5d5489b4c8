"""Rotary positions, head norms with the rotation behind them, and their gradients through the C ABI, against fp64.

Results are fp32, rounded once to bf16: half a step, 2^-8 of the value, or 2^-134 where bf16 is subnormal.  The fp32 part, S the sum of the
magnitudes of a result's terms: cosine and sine to 2 steps each and what the angle loses in fp64 (2^-51 of the turns: 2^-20 at 10^9 and a
frequency of 1), the factor, two products and an addition, within 8 * 2^-24 S (+ 2^-17 S far out: 2 pi 2^-20); a norm's sum of dim squares, its
root and two products add (dim / 2 + 8) * 2^-24 S, the gradients' second sum as much again and 8 roundings.  dgain: a team's heads one after the other,
a wave's teams, four waves, then 16 chains of the workgroups' rows: (chain + 128 + dim) * 2^-24 S."""
import numpy as np
import pytest
import torch

import paper_2511_23225_amd as tw
from oracle import block
from gpu_util import DEV

pytestmark = pytest.mark.gpu
EPS = 1e-6
U = 2.0 ** -24
GUARD = 16.0


def say(*a):
    print(*a, flush=True)


def bf(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16)


def f64(t):
    return t.detach().cpu().double().numpy()


def place(t, how):
    """The heads on the device: by themselves, as a part of a wider tensor, heads in front of tokens, or at an odd address."""
    tokens, heads, dim = t.shape
    if how == "views":
        whole = torch.full((tokens, (heads + 3) * dim), GUARD, dtype=torch.bfloat16, device=DEV)
        v = whole[:, dim:(heads + 1) * dim].unflatten(1, (heads, dim))
    elif how == "turned":
        whole = torch.full((heads, tokens + 1, dim), GUARD, dtype=torch.bfloat16, device=DEV)
        v = whole[:, :tokens].transpose(0, 1)
    elif how == "odd":
        whole = torch.full((tokens * (heads * dim + 5) + 3,), GUARD, dtype=torch.bfloat16, device=DEV)
        v = whole[3:].view(tokens, heads * dim + 5)[:, :heads * dim].unflatten(1, (heads, dim))
    else:
        whole = torch.full((tokens + 1, heads, dim), GUARD, dtype=torch.bfloat16, device=DEV)
        v = whole[:tokens]
    assert v.shape == t.shape
    v.copy_(t)
    return v, whole


def rest_is_untouched(v, whole):
    mark = torch.ones_like(whole, dtype=torch.bool)
    torch.as_strided(mark, v.shape, v.stride(), v.storage_offset()).fill_(False)
    return bool((whole[mark] == GUARD).all())


def inputs(tokens, heads, dim, seed):
    rng = np.random.default_rng(seed)
    n = lambda *s: rng.standard_normal(s)  # noqa: E731
    x = [bf(n(tokens, h, dim)) for h in heads]
    for t in x:
        t.view(-1)[rng.integers(0, t.numel(), 1 + t.numel() // 2000)] = 300.0
    return dict(x=x, dy=[bf(n(tokens, h, dim)) for h in heads], gain=[bf(1 + 0.3 * n(dim)) for _ in heads],
                positions=torch.from_numpy(rng.integers(0, 200000, tokens)))


def freqs_of(rot):
    return tw.tweo_rotary_freqs(rot, kind="turns", factor=4.0, context=8192, low_turns=1.0, high_turns=32.0) if rot else None


def near(got, want, bound, what):
    got = f64(got)
    fine = np.isfinite(want)
    assert (np.isnan(got) == np.isnan(want)).all(), what
    off = np.abs(got - want)[fine]
    lim = (bound + 2.0 ** -8 * np.abs(want) + 2.0 ** -134)[fine]
    worst = float((off / lim).max()) if off.size else 0.0
    assert worst <= 1.0, (what, worst)


# dims of one lane to a team of 32, whole and partly turned, and such that fall between 16-byte pieces or are less than one
DIMS = [(16, 16), (32, 16), (64, 64), (64, 32), (72, 64), (80, 80), (96, 96), (96, 48), (128, 128), (128, 64), (192, 128), (256, 256), (504, 16), (512, 512),
        (8, 8), (20, 20), (64, 20), (33, 10), (2, 2), (3, 2), (100, 100), (510, 510), (511, 4), (17, 16), (18, 18), (24, 18), (40, 34), (98, 66), (130, 96), (259, 100), (500, 484), (505, 34)]
SHAPES = [(1, (1,)), (1, (32, 8)), (3, (5, 3)), (77, (4, 4)), (600, (6, 1))]


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dim,rot", DIMS)
def test_rotary(dim, rot, layout):
    for k, (tokens, heads) in enumerate(SHAPES):
        for how in ("whole", "views", "turned", "odd"):
            scale, transpose = (1.0, False) if k % 2 else (1.25, how == "views")
            say("rotary", tokens, heads, dim, rot, layout, how)
            t = inputs(tokens, heads, dim, k)
            freqs = freqs_of(rot)
            xs = [place(x, how) for x in t["x"]]
            ys = [place(torch.full_like(x, GUARD), how) for x in t["x"]]
            tw.tweo_rotary([(x[0], y[0]) for x, y in zip(xs, ys)], t["positions"].to(DEV), freqs.to(DEV), layout=layout, scale=scale, transpose=transpose)
            torch.cuda.synchronize()
            for x, (y, whole) in zip(t["x"], ys):
                want, size = block.rotary(f64(x), t["positions"].numpy(), freqs.numpy(), layout, scale, transpose)
                near(y, want, 8 * U * size, (tokens, heads, how))
                assert (y[..., rot:].cpu() == x[..., rot:]).all()
                assert rest_is_untouched(y, whole)


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dim,rot", DIMS + [(64, 0), (20, 0)])
def test_norm(dim, rot, layout):
    for k, (tokens, heads) in enumerate(SHAPES):
        for how in ("whole", "views", "odd") if k % 2 else ("turned",):
            say("norm", tokens, heads, dim, rot, layout, how)
            t = inputs(tokens, heads, dim, k + 10)
            freqs, gains = freqs_of(rot), [g if k != 2 else None for g in t["gain"]]
            xs, ys = [place(x, how) for x in t["x"]], [place(torch.full_like(x, GUARD), how) for x in t["x"]]
            turn = dict(positions=t["positions"].to(DEV), freqs=freqs.to(DEV), layout=layout, scale=1.25) if rot else {}
            tw.tweo_head_norm_rotary_fwd([(x[0], None if g is None else g.to(DEV), y[0]) for x, g, y in zip(xs, gains, ys)], eps=EPS, **turn)
            torch.cuda.synchronize()
            for x, g, (y, whole) in zip(t["x"], gains, ys):
                g = np.ones(dim) if g is None else f64(g)
                want, size = block.head_norm_rotary(f64(x), g, EPS, t["positions"].numpy(), freqs.numpy() if rot else None, layout, 1.25)
                near(y, want, (dim / 2 + 16) * U * size, (tokens, heads, how))
                assert rest_is_untouched(y, whole)


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dim,rot", DIMS + [(64, 0), (20, 0)])
def test_grad(dim, rot, layout):
    for k, (tokens, heads) in enumerate(SHAPES):
        for how in ("whole", "views", "odd") if k % 2 else ("turned",):
            say("grad", tokens, heads, dim, rot, layout, how)
            check_grad(tokens, heads, dim, rot, layout, how, k)


def check_grad(tokens, heads, dim, rot, layout, how, k):
    t = inputs(tokens, heads, dim, k + 20)
    freqs, gains = freqs_of(rot), [g if k != 2 else None for g in t["gain"]]
    xs, dys, dxs = ([place(v, how) for v in t[n]] for n in ("x", "dy", "dy"))
    dgains = [torch.full((dim + 8,), 7.0, device=DEV) for _ in heads]
    turn = dict(positions=t["positions"].to(DEV), freqs=freqs.to(DEV), layout=layout, scale=1.25) if rot else {}
    ws = torch.empty(tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, tokens, sum(heads), dim), dtype=torch.uint8, device=DEV)
    groups = [(dy[0], x[0], None if g is None else g.to(DEV), dx[0], dg[:dim] if k != 1 else None) for dy, x, g, dx, dg in zip(dys, xs, gains, dxs, dgains)]
    tw.tweo_head_norm_rotary_bwd(groups, eps=EPS, workspace=ws if k != 1 else None, **turn)
    torch.cuda.synchronize()
    for x, dy, g, (dx, whole), dg, h in zip(t["x"], t["dy"], gains, dxs, dgains, heads):
        g = np.ones(dim) if g is None else f64(g)
        want, dgain, size, gsize = block.head_norm_rotary_bwd(f64(dy), f64(x), g, EPS, t["positions"].numpy(), freqs.numpy() if rot else None, layout, 1.25)
        near(dx, want, (dim + 32) * U * size, (tokens, heads, how))
        assert rest_is_untouched(dx, whole)
        if k != 1:
            assert (np.abs(f64(dg[:dim]) - dgain) <= (tokens * h / 4 + 128 + dim) * U * gsize).all()
        assert (dg[dim if k != 1 else 0:] == 7.0).all()


def test_many_tokens():
    """Several passes over a workgroup's angles, shares of heads and tokens that end anywhere."""
    for tokens, heads, dim, rot in ((20011, (3, 1), 64, 64), (4099, (32, 8), 128, 128), (9001, (1,), 256, 256), (2500, (2, 300), 32, 32), (3, (5000, 1), 64, 64)):
        say("many", tokens, heads, dim)
        check_grad(tokens, heads, dim, rot, "halves", "views", 0)
        t = inputs(tokens, heads, dim, 3)
        freqs = freqs_of(rot)
        y = [torch.empty_like(x, device=DEV) for x in t["x"]]
        tw.tweo_head_norm_rotary_fwd([(x.to(DEV), g.to(DEV), o) for x, g, o in zip(t["x"], t["gain"], y)], t["positions"].to(DEV), freqs.to(DEV), eps=EPS)
        for x, g, o in zip(t["x"], t["gain"], y):
            want, size = block.head_norm_rotary(f64(x), f64(g), EPS, t["positions"].numpy(), freqs.numpy())
            near(o, want, (dim / 2 + 16) * U * size, tokens)


@pytest.mark.parametrize("dim", [64, 20])
def test_far_positions(dim):
    """10^9 with a frequency of 1: the angle keeps 2^-20 of a turn and more."""
    t = inputs(8, (2,), dim, 4)
    pos = torch.tensor([0, 1, 2 ** 20 + 1, 10 ** 9, 10 ** 9 + 1, 2 ** 31 + 5, 7, 3])
    freqs = tw.tweo_rotary_freqs(dim)
    y = torch.empty_like(t["x"][0], device=DEV)
    tw.tweo_rotary([(t["x"][0].to(DEV), y)], pos.to(DEV), freqs.to(DEV))
    want, size = block.rotary(f64(t["x"][0]), pos.numpy(), freqs.numpy())
    near(y, want, (8 * U + 2.0 ** -17) * size, "far")


@pytest.mark.parametrize("norm", [False, True])
def test_most_tokens(norm):
    """2^30 tokens of one head of 2: more workgroups of 64 tokens than a launch holds threads for."""
    tokens, part = 1 << 30, torch.from_numpy(np.random.default_rng(8).standard_normal((1 << 20, 1, 2)).astype(np.float32)).to(torch.bfloat16)
    x = part.to(DEV).repeat(1 << 10, 1, 1)
    pos = torch.arange(tokens, device=DEV).remainder_(100003)
    freqs = tw.tweo_rotary_freqs(2)
    if norm:
        tw.tweo_head_norm_rotary_fwd([(x, None, x)], pos, freqs.to(DEV), eps=EPS)
    else:
        tw.tweo_rotary([(x, x)], pos, freqs.to(DEV))
    for at in (0, 12345, (1 << 28) - 500, (1 << 29) + 77, tokens - 1000):
        src = f64(part[torch.arange(at, at + 1000) % (1 << 20)])
        if norm:
            want, size = block.head_norm_rotary(src, np.ones(2), EPS, pos[at:at + 1000].cpu().numpy(), freqs.numpy(), "halves", 1.0)
        else:
            want, size = block.rotary(src, pos[at:at + 1000].cpu().numpy(), freqs.numpy())
        near(x[at:at + 1000], want, (17 if norm else 8) * U * size, at)


@pytest.mark.parametrize("dim", [64, 20])
def test_padding(dim):
    """Tokens of a negative position: their rows stay as they were, whatever they hold, and count in no gradient."""
    t = inputs(41, (3, 2), dim, 5)
    pad = torch.arange(41) % 3 == 1
    t["positions"][pad] = -1 - torch.arange(int(pad.sum()))
    freqs, pos = freqs_of(dim), t["positions"].numpy()
    keep = ~pad.numpy()
    for v in t["x"] + t["dy"]:
        v[pad] = float("nan")
    dev = lambda name: [v.to(DEV) for v in t[name]]  # noqa: E731
    x, dy, gain, pd, fd = dev("x"), dev("dy"), dev("gain"), t["positions"].to(DEV), freqs.to(DEV)
    out = lambda: [torch.full_like(v, GUARD) for v in x]  # noqa: E731
    y, z, dx, dg = out(), out(), out(), [torch.zeros(dim, device=DEV) for _ in x]
    ws = torch.empty(tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, 41, 5, dim), dtype=torch.uint8, device=DEV)
    tw.tweo_rotary(list(zip(x, y)), pd, fd)
    tw.tweo_head_norm_rotary_fwd(list(zip(x, gain, z)), pd, fd, eps=EPS)
    tw.tweo_head_norm_rotary_bwd(list(zip(dy, x, gain, dx, dg)), pd, fd, eps=EPS, workspace=ws)
    for i in range(2):
        xi, gi, di = f64(t["x"][i])[keep], f64(t["gain"][i]), f64(t["dy"][i])[keep]
        for got in (y[i], z[i], dx[i]):
            assert (got[pad.to(DEV)] == GUARD).all()
        near(y[i][~pad.to(DEV)], *(lambda w, s: (w, 8 * U * s))(*block.rotary(xi, pos[keep], freqs.numpy())), "rotary")
        near(z[i][~pad.to(DEV)], *(lambda w, s: (w, (dim / 2 + 16) * U * s))(*block.head_norm_rotary(xi, gi, EPS, pos[keep], freqs.numpy())), "norm")
        want, dgain, size, gsize = block.head_norm_rotary_bwd(di, xi, gi, EPS, pos[keep], freqs.numpy())
        near(dx[i][~pad.to(DEV)], want, (dim + 32) * U * size, "grad")
        assert (np.abs(f64(dg[i]) - dgain) <= (256 + dim) * U * gsize).all()
    # nothing but padding
    before = [v.clone() for v in y]
    tw.tweo_rotary(list(zip(x, y)), torch.full_like(pd, -7), fd)
    tw.tweo_head_norm_rotary_bwd(list(zip(dy, x, gain, dx, dg)), torch.full_like(pd, -7), fd, eps=EPS, workspace=ws)
    assert all((a == b).logical_or(a.isnan() & b.isnan()).all() for a, b in zip(before, y)) and all((d == 0).all() for d in dg)


@pytest.mark.parametrize("dim", [64, 20])
def test_extreme_rows(dim):
    """Squares beyond fp32 and below it, rows of zeros, infinities and NaN: each head by itself."""
    rng = np.random.default_rng(6)
    x = rng.standard_normal((9, 1, dim))
    x[0] *= 1e30
    x[1] *= 1e-25
    x[2] = 0.0
    x[3, 0, 5] = np.inf
    x[4, 0, 6] = np.nan
    x[5] *= 2.0 ** 49
    x[6] = 3.3e38
    x[7] *= 1e-6
    x = bf(x)
    g = torch.ones(dim, dtype=torch.bfloat16)
    for eps in (1e-6, 0.0):
        y = torch.empty_like(x, device=DEV)
        tw.tweo_head_norm_rotary_fwd([(x.to(DEV), g.to(DEV), y)], eps=eps)
        want = block.head_norm(f64(x), 1.0, eps)
        near(y, want, (dim / 2 + 16) * U * np.where(np.isfinite(want), np.abs(want), 0), eps)


def test_in_place_and_inside_one_tensor():
    """Queries and keys in a qkv tensor, each turned where it lies, side by side or head by head: as out of place, the rest as it was."""
    for tokens, q, k, dim in ((33, 6, 2, 64), (1, 4, 4, 128), (5, 3, 3, 10)):
        qkv = bf(np.random.default_rng(7).standard_normal((tokens, (q + 2 * k) * dim))).to(DEV)
        parts = lambda t: [t[:, :q * dim].unflatten(1, (q, dim)), t[:, q * dim:(q + k) * dim].unflatten(1, (k, dim))]  # noqa: E731
        pos, f = torch.arange(tokens, device=DEV) * 17, tw.tweo_rotary_freqs(dim).to(DEV)
        out = [torch.empty(p.shape, dtype=p.dtype, device=DEV) for p in parts(qkv)]
        tw.tweo_rotary(list(zip(parts(qkv), out)), pos, f)
        own = qkv.clone()
        tw.tweo_rotary([(p, p) for p in parts(own)], pos, f)
        assert all((a == b).all() for a, b in zip(parts(own), out)) and (own[:, (q + k) * dim:] == qkv[:, (q + k) * dim:]).all()
        gain = [bf(np.linspace(0.5, 1.5, dim)).to(DEV)] * 2
        tw.tweo_head_norm_rotary_fwd(list(zip(parts(qkv), gain, out)), pos, f)
        own = qkv.clone()
        tw.tweo_head_norm_rotary_fwd([(p, g, p) for p, g in zip(parts(own), gain)], pos, f)
        assert all((a == b).all() for a, b in zip(parts(own), out))
        # gradients in place of the incoming ones, or of the input
        ws = torch.empty(tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, tokens, q + k, dim), dtype=torch.uint8, device=DEV)
        dqkv, dg = torch.randn_like(qkv), [torch.empty(dim, device=DEV) for _ in range(2)]
        tw.tweo_head_norm_rotary_bwd(list(zip(parts(dqkv), parts(qkv), gain, out, dg)), pos, f, workspace=ws)
        first = [d.clone() for d in dg]
        for target in ("dy", "x"):
            d, x = dqkv.clone(), qkv.clone()
            tw.tweo_head_norm_rotary_bwd(list(zip(parts(d), parts(x), gain, parts(d if target == "dy" else x), dg)), pos, f, workspace=ws)
            assert all((a == b).all() for a, b in zip(parts(d if target == "dy" else x), out))
            assert all((a == b).all() for a, b in zip(dg, first))
    # a part of each head turned, the rest untouched, in place and back
    t = bf(np.random.default_rng(10).standard_normal((21, 3, 96))).to(DEV)
    pos, f, own = torch.arange(21, device=DEV), tw.tweo_rotary_freqs(48).to(DEV), t.clone()
    for layout in ("halves", "pairs"):
        tw.tweo_rotary([(own, own)], pos, f, layout=layout)
        assert (own[..., 48:] == t[..., 48:]).all() and not (own[1:, :, :48] == t[1:, :, :48]).all()
        tw.tweo_rotary([(own, own)], pos, f, layout=layout, transpose=True)
        assert ((own.float() - t.float()).abs() <= 2.0 ** -7 * t.float().abs().amax(-1, keepdim=True)).all()
        own.copy_(t)
    # heads of queries and keys in turn
    t = bf(np.random.default_rng(8).standard_normal((19, 5, 2, 32))).to(DEV)
    pos, f = torch.arange(19, device=DEV), tw.tweo_rotary_freqs(32).to(DEV)
    out = [torch.empty((19, 5, 32), dtype=t.dtype, device=DEV) for _ in range(2)]
    tw.tweo_rotary([(t[:, :, i], out[i]) for i in range(2)], pos, f)
    tw.tweo_rotary([(t[:, :, i], t[:, :, i]) for i in range(2)], pos, f)
    assert all((t[:, :, i] == out[i]).all() for i in range(2))


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dim,rot", [(98, 66), (40, 34), (100, 100), (17, 16), (130, 96), (259, 100)])
def test_in_place_of_odd_widths(dim, rot, layout):
    """Heads whose pieces overlap, where they lie: every call as out of place, bit by bit and again."""
    rng = np.random.default_rng(12)
    x, dy = (bf(rng.standard_normal((701, 7, dim))).to(DEV) for _ in range(2))
    gain = bf(1 + 0.3 * rng.standard_normal(dim)).to(DEV)
    turn = dict(positions=torch.arange(701, device=DEV) * 31, freqs=tw.tweo_rotary_freqs(rot).to(DEV), layout=layout)
    ws = torch.empty(tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, 701, 7, dim), dtype=torch.uint8, device=DEV)
    outs = [torch.empty_like(x) for _ in range(3)]
    dgain, again = torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    tw.tweo_rotary([(x, outs[0])], **turn)
    tw.tweo_head_norm_rotary_fwd([(x, gain, outs[1])], **turn)
    tw.tweo_head_norm_rotary_bwd([(dy, x, gain, outs[2], dgain)], workspace=ws, **turn)
    for _ in range(3):
        own = x.clone()
        tw.tweo_rotary([(own, own)], **turn)
        assert torch.equal(own, outs[0])
        own = x.clone()
        tw.tweo_head_norm_rotary_fwd([(own, gain, own)], **turn)
        assert torch.equal(own, outs[1])
        own = x.clone()
        tw.tweo_head_norm_rotary_bwd([(dy, own, gain, own, again)], workspace=ws, **turn)
        assert torch.equal(own, outs[2]) and torch.equal(again, dgain)
        own = dy.clone()
        tw.tweo_head_norm_rotary_bwd([(own, x, gain, own, again)], workspace=ws, **turn)
        assert torch.equal(own, outs[2]) and torch.equal(again, dgain)


def test_strides_beyond_32_bits():
    """Two tokens, or two heads, more than 2^32 bytes apart."""
    whole = torch.zeros((1 << 31) + (1 << 28) + 256, dtype=torch.bfloat16, device=DEV)
    x = bf(np.random.default_rng(9).standard_normal((2, 2, 64))).to(DEV)
    far = (1 << 31) + (1 << 28)
    pos, f = torch.tensor([3, 5], device=DEV), tw.tweo_rotary_freqs(64).to(DEV)
    want = torch.empty_like(x)
    tw.tweo_rotary([(x, want)], pos, f)
    for strides in ((far, 64, 1), (64, far, 1)):
        v = torch.as_strided(whole, (2, 2, 64), strides)
        v.copy_(x)
        y = torch.empty_like(x)
        tw.tweo_rotary([(v, y)], pos, f)
        tw.tweo_rotary([(v, v)], pos, f)
        assert (y == want).all() and (v == want).all()
        v.zero_()


def test_other_stream_and_graph():
    """On a stream of its own, and captured: replays with other data in the same buffers, eager calls and graphs of the same buffers in between."""
    tokens, q, k, dim = 65, 6, 2, 64
    t = [inputs(tokens, (q, k), dim, s) for s in range(3)]
    f = freqs_of(dim).to(DEV)
    x, dy, gain = ([torch.empty_like(v, device=DEV) for v in t[0][n]] for n in ("x", "dy", "gain"))
    pos = torch.empty_like(t[0]["positions"], device=DEV)
    y, dx = ([torch.zeros_like(v) for v in x] for _ in range(2))
    dg = [torch.zeros(dim, device=DEV) for _ in x]
    ws = [torch.empty(tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, tokens, q + k, dim), dtype=torch.uint8, device=DEV) for _ in range(2)]

    def load(s):
        for a, n in ((x, "x"), (dy, "dy"), (gain, "gain")):
            for d, v in zip(a, s[n]):
                d.copy_(v)
        pos.copy_(s["positions"])

    def step(w):
        tw.tweo_head_norm_rotary_fwd(list(zip(x, gain, y)), pos, f, eps=EPS)
        tw.tweo_head_norm_rotary_bwd(list(zip(dy, x, gain, dx, dg)), pos, f, eps=EPS, workspace=w)
        tw.tweo_rotary([(y[0], y[0])], pos, f, transpose=True)

    def result():
        torch.cuda.synchronize()
        return [v.clone() for v in y + dx + dg]

    eager = []
    for s in t:
        load(s)
        step(ws[0])
        eager.append(result())
    side = torch.cuda.Stream()
    load(t[1])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(ws[1])
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(result(), eager[1]))
    graphs = []
    for w in ws:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(w)
        graphs.append(g)
    for round_ in range(2):
        for i, s in enumerate(t):
            for g in graphs:
                load(s)
                g.replay()
                assert all(torch.equal(a, b) for a, b in zip(result(), eager[i])), (round_, i)
            load(t[(i + 1) % 3])
            step(ws[0])
            assert all(torch.equal(a, b) for a, b in zip(result(), eager[(i + 1) % 3]))


def test_binding_refusals():
    x = torch.zeros((4, 2, 16), dtype=torch.bfloat16, device=DEV)
    y, pos, f = torch.empty_like(x), torch.arange(4, device=DEV), tw.tweo_rotary_freqs(16).to(DEV)
    good = dict(groups=[(x, y)], positions=pos, freqs=f)
    for k in (dict(groups=[]), dict(groups=[(x, y)] * 3), dict(groups=[(x, y, y)]), dict(groups=[(x[:, :, ::2], y[:, :, ::2])]), dict(groups=[(x.float(), y)]),
              dict(groups=[(x, y[:, :1])]), dict(groups=[(x.cpu(), y)]), dict(groups=[(x, y), (x[:2], y[:2])]), dict(groups=[(x[0], y[0])]),
              dict(positions=pos.int()), dict(positions=pos[:3]), dict(positions=None), dict(freqs=f.float()), dict(freqs=None), dict(freqs=f.cpu()),
              dict(freqs=f[::2]), dict(layout="other"), dict(positions=None, freqs=None)):
        with pytest.raises(ValueError):
            tw.tweo_rotary(**{**good, **k})
    with pytest.raises(tw.TweoError):
        tw.tweo_rotary(**{**good, "freqs": tw.tweo_rotary_freqs(18).to(DEV)})
    g = torch.ones(16, dtype=torch.bfloat16, device=DEV)
    for gain in (g.float(), g[:8], g.cpu()):
        with pytest.raises(ValueError):
            tw.tweo_head_norm_rotary_fwd([(x, gain, y)], pos, f)
    dg, ws = torch.empty(16, device=DEV), torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    for group in ((x, x, g, y, dg.double()), (x, x, g, y, dg[:8]), (x, x, g.cpu(), y, dg), (x, x, g, y.float(), dg)):
        with pytest.raises(ValueError):
            tw.tweo_head_norm_rotary_bwd([group], pos, f, workspace=ws)
    with pytest.raises(tw.TweoError):
        tw.tweo_head_norm_rotary_bwd([(x, x, g, y, dg)], pos, f)
    assert tw.tweo_head_norm_rotary_bwd([(x, x, g, y, None)], pos, f) is None
    # one token: whatever its stride says
    one = torch.as_strided(x, (1, 2, 16), (-0, 16, 1))
    tw.tweo_rotary([(one, y[:1])], pos[:1], f)
