"""What a transformer block runs between its 8-bit linears, as cases that can be timed and compared.

  rotary          rotation of queries and keys by their positions
  head_norm       norm of each query and key head and its rotation in one pass
  head_norm_grad  its gradients: of queries and keys, of the two gains
  gated           the gated feed-forward's both FP8 projections, activation and product
  gated_grad      its gradients: of gate and up projection (cast to 8 bits), of the input, of the stacked weight
  w8a8_gated      the gated feed-forward's first half on INT8 operands, for inference

`run` computes them in elementary torch operations or, where `own` is set, by the package's entry points.
"""
import math

import torch

own = False
DEV = "cuda:0"
EPS = 1e-6                          # of the head norms
CONTEXT, FACTOR = 8192, 4.0         # scaled frequencies: a context of so many positions, stretched
SCALE = 1.125                       # what then multiplies the rotated part


def listed():
    return [
        # One token's queries and keys far into a context, half of each head rotated: latency.
        dict(name="rotary-1x40x64", op="rotary", tokens=1, q=32, k=8, dim=64, rot=32, layout="pairs", scaled=False, views=True),
        # Queries and keys of a LLaMA-1B-wide block (16384 tokens) as they lie in the output of its qkv linear.
        dict(name="rotary-16384x32x128", op="rotary", tokens=16384, q=16, k=16, dim=128, rot=128, layout="halves", scaled=True, views=True),
        # One token for each of 64 sequences at a 7B model's width.
        dict(name="head-norm-64x64x128", op="head_norm", tokens=64, q=32, k=32, dim=128, rot=128, layout="halves", scaled=False, views=True, gain=True),
        # The LLaMA-1B-wide block in training.
        dict(name="head-norm-16384x64x64", op="head_norm", tokens=16384, q=32, k=32, dim=64, rot=64, layout="halves", scaled=False, views=True, gain=True),
        # A short ragged batch, heads of a width that fills no power of two, keys shared by three query heads each.
        dict(name="head-norm-grad-513x16x96", op="head_norm_grad", tokens=513, q=12, k=4, dim=96, rot=96, layout="pairs", scaled=True, views=False, gain=True),
        # The LLaMA-1B-wide block in training.
        dict(name="head-norm-grad-16384x64x64", op="head_norm_grad", tokens=16384, q=32, k=32, dim=64, rot=64, layout="halves", scaled=False, views=True, gain=True),
        # A short prompt through a small layer whose sizes fit no tile.
        dict(name="gated-300x528x1000", op="gated", m=300, k=528, f=1000, act="gelu", keep=False),
        # Gate and up projection of the LLaMA-1B block, kept for the backward pass.
        dict(name="gated-16384x2048x5632", op="gated", m=16384, k=2048, f=5632, act="silu", keep=True),
        # A GPT-2-small-wide layer over 1024 tokens, gradients in E5M2.
        dict(name="gated-grad-1024x768x2048", op="gated_grad", m=1024, k=768, f=2048, act="gelu", e5m2=True),
        # The LLaMA-1B block.
        dict(name="gated-grad-16384x2048x5632", op="gated_grad", m=16384, k=2048, f=5632, act="silu", e5m2=False),
        # One token through a 7B model's gate and up projection.
        dict(name="w8a8-gated-1x4096x11008", op="w8a8_gated", m=1, k=4096, f=11008, act="silu", token_steps=True, channel_steps=True),
        # A prompt of 2048 tokens through the same.
        dict(name="w8a8-gated-2048x4096x11008", op="w8a8_gated", m=2048, k=4096, f=11008, act="silu", token_steps=True, channel_steps=True),
    ]


def _log_int(rng, lo, hi, step=1):
    n = round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi)))))
    return max(lo, min(hi, n)) // step * step or step


def draw(rng):
    op = rng.choice(["rotary", "head_norm", "head_norm_grad", "gated", "gated_grad", "w8a8_gated"])
    if op in ("rotary", "head_norm", "head_norm_grad"):
        # most heads are 64, 96 or 128 wide and rotated whole, some are neither
        dim = rng.choice([64, 96, 128]) if rng.random() < 0.6 else 2 * _log_int(rng, 8, 128)
        rot = dim if rng.random() < 0.6 else 2 * rng.randint(1, dim // 2)
        k = _log_int(rng, 1, 32)
        q = k * rng.choice([1, 1, 2, 3, 4]) if k <= 8 else k
        case = dict(op=op, tokens=_log_int(rng, 1, min(32768, (1 << 26) // ((q + k) * dim))), q=q, k=k, dim=dim, rot=rot,
                    layout=rng.choice(["halves", "pairs"]), scaled=rng.random() < 0.4, views=rng.random() < 0.5)
        return case if op == "rotary" else {**case, "gain": rng.random() < 0.8}
    act = rng.choice(["silu", "gelu"])
    if op == "w8a8_gated":
        k = _log_int(rng, 256, 8192, 16)
        f = _log_int(rng, 256, 14336, 8)
        return dict(op=op, m=_log_int(rng, 1, min(4096, 2048 * 4096 * 11008 // (k * f))), k=k, f=f, act=act,
                    token_steps=rng.random() < 0.6, channel_steps=rng.random() < 0.6)
    k, f = _log_int(rng, 128, 4096, 16), _log_int(rng, 128, 8192, 8)
    if rng.random() < 0.5:  # most layers are round
        k, f = -(-k // 128) * 128, -(-f // 128) * 128
    most = min(16384, 16384 * 2048 * 5632 // (k * f))
    if op == "gated":
        return dict(op=op, m=_log_int(rng, 1, most), k=k, f=f, act=act, keep=rng.random() < 0.6)
    return dict(op=op, m=_log_int(rng, 16, most, 16), k=k, f=f, act=act, e5m2=rng.random() < 0.4)


# ------------------------------------------------------------------------------------ inputs
def _gen(seed, index):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1009 + index) & 0x7FFFFFFFFFFF)
    return g


def _normal(shape, std, seed, index):
    return torch.randn(shape, generator=_gen(seed, index), device=DEV) * std


def _frequencies(case):
    """Radians a position, in 64 bits; scaled: slow ones by FACTOR, quick ones not, by their turns over the context in between."""
    f = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=DEV) / case["rot"])
    if case["scaled"]:
        part = ((CONTEXT * f / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
        f = f * (part + (1 - part) / FACTOR)
    return f


def _heads_inputs(case, seed):
    """Queries and keys of a qkv linear, some in extreme channels, each token at its place in one of a few sequences."""
    t, q, k, dim = case["tokens"], case["q"], case["k"], case["dim"]
    width = (q + 2 * k) * dim
    qkv = _normal((t, width), 1.0, seed, 0)
    qkv[:, torch.randint(0, width, (3,), generator=_gen(seed, 1), device=DEV)] *= 30.0
    qkv = qkv.bfloat16()
    parts = (qkv[:, :q * dim].unflatten(1, (q, dim)), qkv[:, q * dim:(q + k) * dim].unflatten(1, (k, dim)))
    s = dict(x=[p if case["views"] else p.contiguous() for p in parts], freqs=_frequencies(case))
    length = max(1, t // 4)
    start = torch.randint(0, 1 << 17, (1,), generator=_gen(seed, 2), device=DEV)
    s["positions"] = torch.arange(t, device=DEV) % length + (start if t < 256 else start // 4096)
    if case["op"] != "rotary":
        s["gain"] = [(1 + _normal((dim,), 0.2, seed, 3 + i)).bfloat16() if case["gain"] else None for i in range(2)]
    if case["op"] == "head_norm_grad":
        s["dy"] = [_normal((t, n, dim), 1.0, seed, 5 + i).bfloat16() for i, n in enumerate((q, k))]
    return s


def _codes(x):
    """Codes and (amax, scale, its inverse) of a bf16 tensor's cast to E4M3 with one scale."""
    amax = x.abs().max().float()
    scale = 448.0 / amax
    q = (x.float() * scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return q, torch.stack([amax, scale, 1.0 / scale])


def _gated_inputs(case, seed):
    """A layer's operands: activations with a few extreme values, weights of deviation 0.02; both projections in one matrix."""
    m, k, f = case["m"], case["k"], case["f"]
    x = _normal((m, k), 1.0, seed, 0)
    x.view(-1)[torch.randint(0, m * k, (m * k // 20000 + 1,), generator=_gen(seed, 1), device=DEV)] *= 8.0
    w = _normal((2 * f, k), 0.02, seed, 2).bfloat16()
    x = x.bfloat16()
    xq, sx = _codes(x)
    wq, sw = _codes(w)
    s = dict(xq=xq, wq=wq, scalars=torch.cat([sx, sw, sx.new_zeros(10)]))
    if case["op"] == "gated_grad":
        s["gu"] = _normal((m, 2 * f), 1.0, seed, 3).bfloat16()
        s["dh"] = _normal((m, f), 1e-3, seed, 4).bfloat16()
    return s


def _w8a8_inputs(case, seed):
    m, k, f = case["m"], case["k"], case["f"]
    x = _normal((m, k), 1.0, seed, 0).clamp(-20.0, 20.0)
    w = _normal((2 * f, k), 0.02, seed, 1)
    s = {}
    for name, t, rows in (("x", x, case["token_steps"]), ("w", w, case["channel_steps"])):
        step = (t.abs().amax(1) if rows else t.abs().max().reshape(1)) / 127.0
        s[name + "q"], s[name + "_step"] = (t / step[:, None]).round().clamp(-127, 127).to(torch.int8), step
    return s


def _inputs(case, seed):
    if case["op"] in ("rotary", "head_norm", "head_norm_grad"):
        return _heads_inputs(case, seed)
    return _w8a8_inputs(case, seed) if case["op"] == "w8a8_gated" else _gated_inputs(case, seed)


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    empty = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    bf = lambda *shape: empty(shape, torch.bfloat16)  # noqa: E731
    if "x" in s:
        s["y"] = [bf(*x.shape) for x in s["x"]]
        if case["op"] == "head_norm_grad":
            s["dgain"] = [empty((case["dim"],), torch.float32) if g is not None else None for g in s["gain"]]
            if own:
                import paper_2511_23225_amd as tw
                s["workspace"] = empty((tw.tweo_workspace_bytes(tw.TWEO_OP_HEAD_NORM_ROTARY_BWD, case["tokens"], case["q"] + case["k"], case["dim"]),), torch.uint8)
        return s
    m, k, f = case["m"], case["k"], case["f"]
    if case["op"] != "gated_grad":
        s["h"] = bf(m, f)
        if case["op"] == "gated":
            s["gu"] = bf(m, 2 * f) if case["keep"] else None
        return s
    s.update(dx=bf(m, k), dw=bf(2 * f, k), dguq=empty((m, 2 * f), torch.uint8))
    s["xqT"], s["wqT"] = (s[n].view(torch.uint8).t().contiguous() for n in ("xq", "wq"))  # the forward pass has left them
    if own:
        import paper_2511_23225_amd as tw
        s["saved"] = tw.make_saved(s["xq"], s["xqT"], s["wq"], s["wqT"], s["scalars"])
        s["dguqT"] = empty((2 * f, m), torch.uint8)
        s["workspace"] = empty((tw.tweo_workspace_bytes(tw.TWEO_OP_FP8_GATED_BWD_BF16, m, f, k),), torch.uint8)
    return s


# ------------------------------------------------------------------------------- the plain forms
def _turned(x, cos, sin, case):
    """x [tokens, heads, dim] with its first `rot` values turned by the angles' cosines and sines [tokens, rot / 2]."""
    rot = case["rot"]
    cos, sin = cos[:, None], sin[:, None]
    if case["layout"] == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., rot:]], -1)


def _angles(s):
    angle = s["positions"].double()[:, None] * s["freqs"]
    scale = SCALE if s["case"]["scaled"] else 1.0
    return (angle.cos() * scale).float(), (angle.sin() * scale).float()


def _plain_heads(s):
    c = s["case"]
    cos, sin = _angles(s)
    for i, x in enumerate(s["x"]):
        x = x.float()
        if c["op"] == "rotary":
            s["y"][i].copy_(_turned(x, cos, sin, c))
            continue
        gain = 1.0 if s["gain"][i] is None else s["gain"][i].float()
        rstd = 1 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        if c["op"] == "head_norm":
            s["y"][i].copy_(_turned(x * rstd * gain, cos, sin, c))
            continue
        dy, xhat = _turned(s["dy"][i].float(), cos, -sin, c), x * rstd
        w = dy * gain
        s["y"][i].copy_(rstd * (w - xhat * (w * xhat).mean(-1, keepdim=True)))
        if s["dgain"][i] is not None:
            s["dgain"][i].copy_((dy * xhat).sum((0, 1)))


def _share(g, act):
    """The activation over its argument and the derivative of what goes into the sigmoid."""
    if act == "silu":
        return 1 / (1 + (-g).exp()), 1.0
    z = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g)
    return 1 / (1 + (-z).exp()), 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)


def _plain_gated(s):
    f, act = s["case"]["f"], s["case"]["act"]
    gu = s["xq"].float() @ s["wq"].float().t() * (s["scalars"][2] * s["scalars"][5])
    gu = gu.bfloat16()  # as the layer stores them and its backward pass reads them
    if s["gu"] is not None:
        s["gu"].copy_(gu)
    g, u = gu[:, :f].float(), gu[:, f:].float()
    s["h"].copy_(g * _share(g, act)[0] * u)


def _plain_gated_grad(s):
    c = s["case"]
    f, kind, top = c["f"], torch.float8_e5m2 if c["e5m2"] else torch.float8_e4m3fn, 57344.0 if c["e5m2"] else 448.0
    g, u, dh = s["gu"][:, :f].float(), s["gu"][:, f:].float(), s["dh"].float()
    part, slope = _share(g, c["act"])
    dgu = torch.cat([dh * u * (part + g * part * (1 - part) * slope), dh * g * part], 1).bfloat16().float()
    scale = top / dgu.abs().max()
    q = (dgu * scale).clamp(-top, top).to(kind)
    s["dguq"].copy_(q.view(torch.uint8))
    q = q.float()
    s["dx"].copy_(q @ s["wq"].float() * (s["scalars"][5] / scale))
    s["dw"].copy_(q.t() @ s["xq"].float() * (s["scalars"][2] / scale))


def _plain_w8a8(s):
    f = s["case"]["f"]
    # whole numbers beyond 2^24
    acc = s["xq"].double() @ s["wq"].double().t()
    gu = acc.float() * s["x_step"][:, None] * s["w_step"]
    g, u = gu[:, :f], gu[:, f:]
    s["h"].copy_(g * _share(g, s["case"]["act"])[0] * u)


def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2511_23225_amd as tw
    if c["op"] in ("rotary", "head_norm", "head_norm_grad"):
        if own:
            turn = dict(layout=c["layout"], scale=SCALE if c["scaled"] else 1.0)
            if c["op"] == "rotary":
                tw.tweo_rotary(list(zip(s["x"], s["y"])), s["positions"], s["freqs"], **turn)
            elif c["op"] == "head_norm":
                tw.tweo_head_norm_rotary_fwd(list(zip(s["x"], s["gain"], s["y"])), s["positions"], s["freqs"], eps=EPS, **turn)
            else:
                tw.tweo_head_norm_rotary_bwd(list(zip(s["dy"], s["x"], s["gain"], s["y"], s["dgain"])), s["positions"], s["freqs"], eps=EPS,
                                             workspace=s["workspace"], **turn)
        else:
            _plain_heads(s)
        return dict(q=s["y"][0], k=s["y"][1], gains=s.get("dgain"))
    if c["op"] == "gated":
        if own:
            tw.tweo_fp8_gated_fwd(s["xq"].view(torch.uint8), s["scalars"][2:3], s["wq"].view(torch.uint8), s["scalars"][5:6], s["h"], gu_bf16=s["gu"],
                                  act=c["act"])
        else:
            _plain_gated(s)
        return dict(h=s["h"], gu=s["gu"])
    if c["op"] == "gated_grad":
        if own:
            tw.tweo_fp8_gated_bwd_bf16(s["dh"], s["gu"], s["saved"], c["k"], s["dguq"], s["dguqT"], dx_bf16=s["dx"], dw_bf16=s["dw"], act=c["act"],
                                       dy_e5m2=c["e5m2"], workspace=s["workspace"])
        else:
            _plain_gated_grad(s)
        return dict(dgu=s["dguq"].view(torch.float8_e5m2 if c["e5m2"] else torch.float8_e4m3fn), dx=s["dx"], dw=s["dw"])
    if own:
        tw.tweo_w8a8_gated(s["xq"], s["wq"], s["x_step"], s["w_step"], s["h"], act=c["act"])
    else:
        _plain_w8a8(s)
    return s["h"]


def work(case):
    if case["op"] in ("rotary", "head_norm", "head_norm_grad"):
        n, t = case["tokens"] * (case["q"] + case["k"]) * case["dim"], case["tokens"]
        once = 8 * t + 4 * case["rot"]
        if case["op"] == "rotary":
            return dict(bytes=4 * n + once, flops=3.0 * n * case["rot"] / case["dim"])
        gains = 2 * case["dim"] * case["gain"]
        if case["op"] == "head_norm":
            return dict(bytes=4 * n + once + 2 * gains, flops=7.0 * n)
        return dict(bytes=6 * n + once + 6 * gains, flops=13.0 * n)
    m, k, f = case["m"], case["k"], case["f"]
    product = 2.0 * m * k * 2 * f
    if case["op"] == "gated":
        return dict(bytes=m * k + 2 * f * k + 2 * m * f * (3 if case["keep"] else 1), flops=product)
    if case["op"] == "gated_grad":
        return dict(bytes=m * f * 6 + 2 * m * f + 2 * f * k + m * k + 2 * m * k + 4 * f * k, flops=2 * product)
    return dict(bytes=m * k + 2 * f * k + 2 * m * f + 4 * (m if case["token_steps"] else 1) + 4 * (2 * f if case["channel_steps"] else 1), flops=product)


# -------------------------------------------------------------------------- the same in 64 bits
def _spin64(x, positions, freqs, factor, layout, sign):
    """Each pair as a complex number, times factor * exp(i * angle)."""
    n = freqs.numel()
    turn = torch.polar(torch.full((positions.numel(), n), factor, dtype=torch.float64, device=DEV), sign * torch.outer(positions.to(torch.float64), freqs))
    head, rest = x[..., :2 * n], x[..., 2 * n:]
    pairs = head.unflatten(-1, (2, n)).transpose(-1, -2) if layout == "halves" else head.unflatten(-1, (n, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn.unsqueeze(1))
    z = z.transpose(-1, -2) if layout == "halves" else z
    return torch.cat((z.reshape(head.shape), rest), dim=-1)


def _exact_heads(case, s):
    factor, out, gains = SCALE if case["scaled"] else 1.0, [], []
    for i, x in enumerate(s["x"]):
        x = x.to(torch.float64)
        if case["op"] == "rotary":
            out.append(_spin64(x, s["positions"], s["freqs"], factor, case["layout"], 1.0))
            continue
        gain = torch.ones(case["dim"], dtype=torch.float64, device=DEV) if s["gain"][i] is None else s["gain"][i].to(torch.float64)
        if case["op"] == "head_norm":
            y = x * gain / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / case["dim"] + EPS)
            out.append(_spin64(y, s["positions"], s["freqs"], factor, case["layout"], 1.0))
            continue
        x.requires_grad_()
        gain.requires_grad_()
        y = x * gain / torch.sqrt((x * x).sum(-1, keepdim=True) / case["dim"] + EPS)
        back = _spin64(s["dy"][i].to(torch.float64), s["positions"], s["freqs"], factor, case["layout"], -1.0)
        dx, dgain = torch.autograd.grad((y * back).sum(), (x, gain))
        out.append(dx)
        gains.append(dgain if s["gain"][i] is not None else None)
    return dict(q=out[0], k=out[1], gains=gains if case["op"] == "head_norm_grad" else None)


def _act64(g, act):
    return g * torch.sigmoid(g) if act == "silu" else 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def exact(case, seed):
    s = _inputs(case, seed)
    if "x" in s:
        return _exact_heads(case, s)
    f, act = case["f"], case["act"]
    if case["op"] == "w8a8_gated":
        gate, up = ((s["xq"].to(torch.float64) * s["x_step"].to(torch.float64)[:, None]) @
                    (s["wq"].to(torch.float64) * s["w_step"].to(torch.float64)[:, None]).T).split(f, dim=1)
        return _act64(gate, act) * up
    x = s["xq"].to(torch.float64) * s["scalars"][2].to(torch.float64)
    w = s["wq"].to(torch.float64) * s["scalars"][5].to(torch.float64)
    if case["op"] == "gated":
        gu = torch.mm(x, w.T)
        return dict(h=_act64(gu[:, :f], act) * gu[:, f:], gu=gu if case["keep"] else None)
    gate, up = (t.to(torch.float64).requires_grad_() for t in s["gu"].split(f, dim=1))
    with torch.enable_grad():
        grads = torch.autograd.grad(_act64(gate, act) * up, (gate, up), s["dh"].to(torch.float64))
    stored = torch.hstack(grads).to(torch.bfloat16).to(torch.float64)
    kind = torch.float8_e5m2 if case["e5m2"] else torch.float8_e4m3fn
    scale = (torch.finfo(kind).max / stored.abs().amax().to(torch.float32)).to(torch.float64)
    codes = (stored * scale).clamp(-torch.finfo(kind).max, torch.finfo(kind).max).to(kind).to(torch.float64)
    return dict(dgu=codes, dx=(codes / scale) @ w, dw=(codes / scale).T @ x)
