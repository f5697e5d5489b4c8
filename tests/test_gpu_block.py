"""A transformer block's forward and backward pass through the package's entry points one after the other, as a training step runs them: norm, qkv
linear, norm and rotation of queries and keys in the qkv tensor, (a stand-in for attention,) output linear, norm, gated feed-forward, down linear;
and the INT8 path of the feed-forward as serving runs it.

Against float64 autograd of the same block on the same bf16 weights, without any quantisation.  A cast to E4M3 is off by at most half a step, 2^-4 of a
value, uniformly: 2^-4 / sqrt(3) = 3.6 % in the 2-norm.  A result has at most 16 such casts on its ways (two operands of each of up to eight products),
independent of each other and passed on by maps that do not amplify beside a residual stream: sqrt(16) * 3.6 % = 14.4 %; held to 20 %.  INT8: a
step of 1/127 of a row's largest of K normal numbers, 3.5 to 4.5 deviations: 4.5 / 127 / sqrt(12) = 1 % an operand, four operands and the static
step of h: 2.3 %; held to 4 %."""
import numpy as np
import pytest
import torch

import paper_2511_23225_amd as tw
from gpu_util import DEV

pytestmark = pytest.mark.gpu
EPS = 1e-5


def say(*a):
    print(*a, flush=True)


def b16(*s):
    return torch.zeros(s, dtype=torch.bfloat16, device=DEV)


def u8(*s):
    return torch.empty(s, dtype=torch.uint8, device=DEV)


class Linear:
    """Weight, codes and gradients of an FP8 linear."""

    def __init__(self, M, N, K, gen, gated=False):
        self.M, self.N, self.K, self.gated = M, N, K, gated
        self.w = (torch.randn((N, K), generator=gen) * K ** -0.5).bfloat16().to(DEV)
        self.buf, self.sc = [u8(M, K), u8(K, M), u8(N, K), u8(K, N)], torch.zeros(16, device=DEV)
        self.saved, self.dyq, self.dyqT, self.dw, self.dx = tw.make_saved(*self.buf, self.sc), u8(M, N), u8(N, M), b16(N, K), b16(M, K)
        ops = (tw.TWEO_OP_FP8_GATED_FWD_BF16, tw.TWEO_OP_FP8_GATED_BWD_BF16) if gated else (tw.TWEO_OP_FP8_LINEAR_FWD_BF16, tw.TWEO_OP_FP8_LINEAR_BWD_BF16)
        self.ws = u8(max(tw.tweo_workspace_bytes(op, M, N // 2 if gated else N, K) for op in ops))

    def fwd(self, x, y, residual=None):
        tw.tweo_fp8_linear_fwd_bf16(x, self.w, y, self.saved, residual_bf16=residual, workspace=self.ws)

    def bwd(self, dy):
        tw.tweo_fp8_linear_bwd_bf16(dy, self.saved, self.K, self.dyq, self.dyqT, self.dx, self.dw, workspace=self.ws)
        return self.dx


class Block:
    def __init__(self, M, heads, dim, F, act, layout, seed=0):
        g = torch.Generator().manual_seed(seed)
        W = heads * dim
        self.M, self.heads, self.dim, self.W, self.F, self.act, self.layout = M, heads, dim, W, F, act, layout
        self.qkv, self.o, self.gu, self.down = Linear(M, 3 * W, W, g), Linear(M, W, W, g), Linear(M, 2 * F, W, g, True), Linear(M, W, F, g)
        self.gamma = [(1 + 0.1 * torch.randn(W, generator=g)).bfloat16().to(DEV) for _ in range(2)]
        self.gain = [(1 + 0.1 * torch.randn(dim, generator=g)).bfloat16().to(DEV) for _ in range(2)]
        self.x, self.dy, self.y, self.dx = b16(M, W), b16(M, W), b16(M, W), b16(M, W)
        self.n = [b16(M, W) for _ in range(2)]
        self.stats = [torch.empty((M, 2), dtype=torch.float64, device=DEV) for _ in range(2)]
        self.t, self.turned, self.a, self.mid, self.h, self.kept = b16(M, 3 * W), b16(M, 2 * W), b16(M, W), b16(M, W), b16(M, F), b16(M, 2 * F)
        self.dmid, self.dt, self.dgamma, self.dgain = b16(M, W), b16(M, 3 * W), [torch.empty(W, device=DEV) for _ in range(2)], [torch.empty(dim, device=DEV) for _ in range(2)]
        self.pos, self.freqs = torch.arange(M, device=DEV) % 64, tw.tweo_rotary_freqs(dim // 2 * 2).to(DEV)
        self.ws = u8(max(tw.tweo_workspace_bytes(tw.TWEO_OP_LAYERNORM_BWD, M, W, 1), tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, M, 2 * heads, dim)))

    def parts(self, t):
        return [t[:, i * self.W:(i + 1) * self.W].unflatten(1, (self.heads, self.dim)) for i in range(2)]

    def step(self):
        turn = dict(layout=self.layout, eps=EPS)
        tw.tweo_layernorm_fwd(self.x, self.gamma[0], self.n[0], eps=EPS, stats_out=self.stats[0])
        self.qkv.fwd(self.n[0], self.t)
        tw.tweo_head_norm_rotary_fwd(list(zip(self.parts(self.t), self.gain, self.parts(self.turned))), self.pos, self.freqs, **turn)
        torch.add(self.turned[:, :self.W], self.turned[:, self.W:], out=self.a)  # in attention's place
        self.a += self.t[:, 2 * self.W:]
        self.o.fwd(self.a, self.mid, residual=self.x)
        tw.tweo_layernorm_fwd(self.mid, self.gamma[1], self.n[1], eps=EPS, stats_out=self.stats[1])
        tw.tweo_fp8_gated_fwd_bf16(self.n[1], self.gu.w, self.h, self.kept, self.gu.saved, act=self.act, workspace=self.gu.ws)
        self.down.fwd(self.h, self.y, residual=self.mid)

        dh = self.down.bwd(self.dy)
        gu = self.gu
        tw.tweo_fp8_gated_bwd_bf16(dh, self.kept, gu.saved, gu.K, gu.dyq, gu.dyqT, gu.dx, gu.dw, act=self.act, workspace=gu.ws)
        tw.tweo_layernorm_bwd(gu.dx, self.mid, self.gamma[1], self.stats[1], self.dmid, self.dgamma[1], residual_grad_bf16=self.dy, workspace=self.ws)
        da = self.o.bwd(self.dmid)
        heads = da.unflatten(1, (self.heads, self.dim))
        tw.tweo_head_norm_rotary_bwd([(heads, x, g, dx, dg) for x, g, dx, dg in zip(self.parts(self.t), self.gain, self.parts(self.dt), self.dgain)],
                                     self.pos, self.freqs, workspace=self.ws, **turn)
        self.dt[:, 2 * self.W:].copy_(da)
        tw.tweo_layernorm_bwd(self.qkv.bwd(self.dt), self.x, self.gamma[0], self.stats[0], self.dx, self.dgamma[0], residual_grad_bf16=self.dmid, workspace=self.ws)

    def results(self):
        names = ["y", "dx"] + [n + ".dw" for n in ("qkv", "o", "gu", "down")] + ["dgamma.0", "dgamma.1", "dgain.0", "dgain.1"]
        out = [self.y, self.dx] + [l.dw for l in (self.qkv, self.o, self.gu, self.down)] + self.dgamma + self.dgain
        return dict(zip(names, out))

    def load(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.x.copy_(torch.randn(self.x.shape, generator=g))
        self.dy.copy_(torch.randn(self.dy.shape, generator=g))

    def reference(self):
        d = lambda t: t.detach().cpu().double().requires_grad_()  # noqa: E731
        x, weights, gamma, gain = d(self.x), [d(l.w) for l in (self.qkv, self.o, self.gu, self.down)], [d(g) for g in self.gamma], [d(g) for g in self.gain]
        angle = self.pos.cpu().double()[:, None] * self.freqs.cpu()
        z = torch.polar(torch.ones_like(angle), angle)[:, None]

        def norm(x, g):
            return (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + EPS).sqrt() * g

        def heads(x, g):
            x = x.unflatten(1, (self.heads, self.dim))
            x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * g
            p = x.unflatten(-1, (2, -1)).transpose(-1, -2) if self.layout == "halves" else x.unflatten(-1, (-1, 2))
            p = torch.view_as_real(torch.complex(p[..., 0], p[..., 1]) * z)
            return (p.transpose(-1, -2) if self.layout == "halves" else p).reshape(x.shape).flatten(1)

        t = norm(x, gamma[0]) @ weights[0].T
        q, k, v = t.split(self.W, 1)
        mid = x + (heads(q, gain[0]) + heads(k, gain[1]) + v) @ weights[1].T
        gate, up = (norm(mid, gamma[1]) @ weights[2].T).split(self.F, 1)
        act = torch.nn.functional.silu(gate) if self.act == "silu" else torch.nn.functional.gelu(gate, approximate="tanh")
        y = mid + (act * up) @ weights[3].T
        grads = torch.autograd.grad((y * self.dy.cpu().double()).sum(), [x] + weights + gamma + gain)
        return dict(zip(self.results(), [y.detach()] + list(grads)))


@pytest.mark.parametrize("M,heads,dim,F,act,layout", [(256, 4, 64, 512, "silu", "halves"), (528, 3, 96, 784, "gelu", "pairs"), (1024, 16, 64, 2816, "silu", "halves")])
def test_block_forward_and_backward(M, heads, dim, F, act, layout):
    say("block", M, heads, dim, F)
    block = Block(M, heads, dim, F, act, layout)
    block.load(1)
    block.step()
    torch.cuda.synchronize()
    want = block.reference()
    for name, got in block.results().items():
        got, ref = got.detach().cpu().double(), want[name]
        off = float((got - ref).norm() / ref.norm())
        say("  ", name, round(off, 4))
        assert off <= 0.2, (name, off)


def test_block_in_a_graph():
    """A whole step captured twice, replayed with other data, with eager steps of the same buffers in between."""
    block = Block(272, 2, 64, 272, "silu", "halves")
    eager = []
    for seed in range(3):
        block.load(seed)
        block.step()
        torch.cuda.synchronize()
        eager.append({k: v.clone() for k, v in block.results().items()})
    graphs = []
    side = torch.cuda.Stream()
    for _ in range(2):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            block.step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            block.step()
        graphs.append(g)
    for seed in (1, 0, 2, 1):
        for g in graphs:
            block.load(seed)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(v, eager[seed][k]) for k, v in block.results().items()), seed
        block.load(2 - seed)
        block.step()
        torch.cuda.synchronize()
        assert all(torch.equal(v, eager[2 - seed][k]) for k, v in block.results().items())


@pytest.mark.parametrize("M", [1, 7, 64, 300])
@pytest.mark.parametrize("i8", [False, True])
def test_int8_feed_forward(M, i8):
    """Quantised tokens through gate, up and down projection: h in bf16 and quantised again, or in INT8 under a static step."""
    W, F = 512, 1376
    say("int8 feed-forward", M, i8)
    g = torch.Generator().manual_seed(M)
    x, wgu, wd = (torch.randn(s, generator=g).bfloat16().to(DEV) for s in ((M, W), (2 * F, W), (W, F)))
    wgu, wd = wgu * W ** -0.5, wd * F ** -0.5
    i = lambda *s: torch.empty(s, dtype=torch.int8, device=DEV)  # noqa: E731
    q, sw, qd, sd, xq, sx, hq, y = i(2 * F, W), torch.empty(2 * F, device=DEV), i(W, F), torch.empty(W, device=DEV), i(M, W), torch.empty(M, device=DEV), i(M, F), b16(M, W)
    for t, codes, step in ((wgu, q, sw), (wd, qd, sd), (x, xq, sx)):
        tw.tweo_quantize_i8_rows(t, 0.0, codes, step)
    d = lambda t: t.detach().cpu().double()  # noqa: E731
    gate, up = (d(x) @ d(wgu).T).split(F, 1)
    h = torch.nn.functional.silu(gate) * up
    if i8:
        top = float(h.abs().max())
        tw.tweo_w8a8_gated_i8out(xq, q, sx, sw, 127.0 / top, hq)
        sh = torch.full((1,), top / 127.0, device=DEV)
    else:
        hb, sh = b16(M, F), torch.empty(M, device=DEV)
        tw.tweo_w8a8_gated(xq, q, sx, sw, hb)
        tw.tweo_quantize_i8_rows(hb, 0.0, hq, sh)
    tw.tweo_w8a8_linear_scaled(hq, qd, sh, sd, y)
    want = h @ d(wd).T
    off = float((d(y) - want).norm() / want.norm())
    # a static step of the largest of M * F products is wider than a row's own: h's rms is 0.36, its largest some 12 to 20
    assert off <= (0.04 if not i8 else 0.04 + float(sh) / 12 ** 0.5 / float(h.square().mean().sqrt())), off
