"""Rotary positions and head norms at the ends of what they take, on the GPU, against fp64.  Bounds of single results as in test_gpu_heads.py."""
import numpy as np
import pytest
import torch

import paper_2511_23225_amd as tw
from oracle import block
from gpu_util import DEV
from test_gpu_heads import EPS, U, bf, f64, freqs_of, inputs, near
from test_heads_sums import CASES, gain_steps

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


def test_queries_key_by_key():
    """A qkv tensor that holds each key head's queries, the key and the value one behind the other: a key head of a token as a token."""
    tokens, keys, each, dim = 37, 3, 4, 64
    rng = np.random.default_rng(1)
    host = bf(rng.standard_normal((tokens, keys, each + 2, dim)))
    pos, f, gain = torch.from_numpy(rng.integers(0, 5000, tokens)), freqs_of(dim), bf(1 + 0.3 * rng.standard_normal(dim))
    pos[5] = -1
    qkv, flat = host.to(DEV), pos.to(DEV).repeat_interleave(keys)
    parts = lambda t: (t.view(tokens * keys, each + 2, dim)[:, :each], t.view(tokens * keys, each + 2, dim)[:, each:each + 1])  # noqa: E731
    keep = np.arange(tokens) != 5
    for norm in (False, True):
        own = qkv.clone()
        if norm:
            tw.tweo_head_norm_rotary_fwd([(p, gain.to(DEV), p) for p in parts(own)], flat, f.to(DEV), eps=EPS)
        else:
            tw.tweo_rotary([(p, p) for p in parts(own)], flat, f.to(DEV))
        assert torch.equal(own[5], qkv[5]) and torch.equal(own[:, :, each + 1], qkv[:, :, each + 1])
        for i in range(each + 1):
            x = f64(host[:, :, i])[keep]
            if norm:
                want, size = block.head_norm_rotary(x, f64(gain), EPS, pos.numpy()[keep], f.numpy())
            else:
                want, size = block.rotary(x, pos.numpy()[keep], f.numpy())
            near(own[:, :, i][torch.from_numpy(keep).to(DEV)], want, (dim / 2 + 16 if norm else 8) * U * size, (norm, i))


def grads_of(t, gains, turn, eps, tokens, heads, dim):
    """dx and dgain, with the workspace of as many bytes as are asked for in front of others, which stay as they were."""
    dev = lambda v: v.to(DEV)  # noqa: E731
    need = tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, tokens, sum(heads), dim)
    whole = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    dx = [torch.empty(v.shape, dtype=v.dtype, device=DEV) for v in t["x"]]
    dgain = [torch.full((dim + 8,), 7.0, device=DEV) for _ in heads]
    tw.tweo_head_norm_rotary_bwd([(dev(dy), dev(x), None if g is None else dev(g), o, d[:dim]) for dy, x, g, o, d in zip(t["dy"], t["x"], gains, dx, dgain)],
                                 eps=eps, workspace=whole[:need], **turn)
    torch.cuda.synchronize()
    assert (whole[need:] == 0xA5).all() and all((d[dim:] == 7.0).all() for d in dgain)
    return dx, [f64(d[:dim]) for d in dgain]


@pytest.mark.parametrize("tokens,heads,dim,rot", CASES)
def test_gain_gradients(tokens, heads, dim, rot):
    """Sums over more heads than the workgroups take at a time, to the additions that a term goes through (test_heads_sums.py)."""
    say("gain gradients", tokens, heads, dim, rot)
    t, freqs = inputs(tokens, heads, dim, 31), freqs_of(rot)
    layout = "pairs" if tokens % 2 else "halves"
    turn = dict(positions=t["positions"].to(DEV), freqs=freqs.to(DEV), layout=layout, scale=1.25)
    dx, dgain = grads_of(t, t["gain"], turn, EPS, tokens, heads, dim)
    for i in range(len(heads)):
        args = f64(t["dy"][i]), f64(t["x"][i]), f64(t["gain"][i]), EPS, t["positions"].numpy(), freqs.numpy(), layout, 1.25
        want, total, size, gsize = block.head_norm_rotary_bwd(*args)
        near(dx[i], want, (dim + 32) * U * size, (tokens, heads))
        off = np.abs(dgain[i] - total) / (gain_steps(tokens, heads, i, dim, rot) * U * gsize)
        say("  ", round(float(off.max()), 4))
        assert off.max() <= 1, off.max()


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("tokens,heads,dim,rot", [(20011, (3, 1), 64, 64), (4099, (32, 8), 128, 128), (9001, (1,), 256, 256), (2500, (2, 300), 32, 32), (3, (5000, 1), 64, 64),
                                                  (2777, (3, 5), 512, 512), (30011, (1, 2), 32, 20), (40009, (2,), 8, 8), (50000, (1,), 64, 0), (1, (7, 1), 16, 16), (100003, (1, 1), 16, 16)])
def test_gain_gradients_of_whole_numbers(tokens, heads, dim, rot, layout):
    """Heads of ones and minus ones, whose norm is one to the bit (widths that are powers of two), not turned (positions of 0): the sums of whole numbers
    below 2^24 are exact in any order, and no contribution is lost, counted twice or put elsewhere."""
    say("whole numbers", tokens, heads, dim, rot, layout)
    rng = np.random.default_rng(tokens)
    t = dict(x=[bf(rng.choice([-1.0, 1.0], (tokens, h, dim))) for h in heads], dy=[bf(rng.integers(-9, 10, (tokens, h, dim))) for h in heads])
    turn = dict(positions=torch.zeros(tokens, dtype=torch.int64, device=DEV), freqs=freqs_of(rot).to(DEV), layout=layout) if rot else {}
    _, dgain = grads_of(t, [None] * len(heads), turn, 0.0, tokens, heads, dim)
    for x, dy, d in zip(t["x"], t["dy"], dgain):
        want = (f64(x) * f64(dy)).sum((0, 1))
        assert np.abs(f64(dy)).sum((0, 1)).max() < 2 ** 24 and (d == want).all()


@pytest.mark.parametrize("dim,rot", [(64, 64), (20, 0), (98, 66), (7, 4)])
@pytest.mark.parametrize("eps", [1e-6, 1e-30, 0.0])
def test_gradients_of_extreme_rows(dim, rot, eps):
    """Heads whose squares leave fp32 at either end (to the least root mean square that has an fp32 reciprocal), gradients to match; zeros, infinities and
    NaN spoil their own head, and dgain what the formula says."""
    say("gradients of extreme rows", dim, rot, eps)
    rng = np.random.default_rng(11)
    x, dy = rng.standard_normal((13, 1, dim)), rng.standard_normal((13, 1, dim))
    x[0] *= 1e30
    x[1] *= 1e-25
    x[2] *= 2.0 ** 49
    x[3] = rng.choice([-3.3e38, 3.3e38], (1, dim))
    x[4] *= 1e-6
    x[5] *= 1e30
    dy[5] *= 1e28
    x[6] *= 2.0 ** -41  # squares about the border of the second way
    x[7] *= 1e-14
    x[8] = rng.choice([-4e-39, 4e-39], (1, dim))
    dy[8] *= 0.05
    finite = 9
    x[9] = 0.0
    x[10, 0, dim // 2] = np.inf
    x[11, 0, dim - 1] = np.nan
    dy[12, 0, 0] = np.nan
    x, dy, g = bf(x), bf(dy), bf(1 + 0.3 * rng.standard_normal(dim))
    pos, f = torch.from_numpy(rng.integers(0, 1000, 13)), freqs_of(rot)

    def both(n):
        turn = dict(positions=pos[:n].to(DEV), freqs=f.to(DEV), layout="pairs") if rot else {}
        dx, dgain = grads_of(dict(x=[x[:n]], dy=[dy[:n]]), [g], turn, eps, n, (1,), dim)
        return dx[0], dgain[0], block.head_norm_rotary_bwd(f64(dy[:n]), f64(x[:n]), f64(g), float(np.float32(eps)), pos.numpy()[:n], f.numpy() if rot else None, "pairs", 1.0)

    dx, dgain, (want, total, size, gsize) = both(finite)
    assert np.isfinite(want).all() and np.abs(want).max() < 3e38
    near(dx, want, (dim + 32) * U * size, eps)
    assert (np.abs(dgain - total) <= gain_steps(finite, (1,), 0, dim, rot) * U * gsize).all()
    dx, dgain, (want, total, size, gsize) = both(13)
    near(dx, want, (dim + 32) * U * np.nan_to_num(size), eps)
    assert (np.isnan(dgain) == np.isnan(total)).all()
