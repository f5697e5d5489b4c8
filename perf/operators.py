"""What stands between the FP8 linears' gradients and the next step's weights, as cases that can be timed and compared.

  layernorm_fwd   residual add + LayerNorm to bf16, with the row statistics that a backward pass takes
  layernorm_bwd   its gradients: of the row (with the gradient that reaches the stream past the norm), of gain and bias
  sumsq           the sum of the squares of all gradients, for clipping by their global norm
  adamw           an AdamW step over all tensors of a model, states in 32 or in 8 bits

`run` computes them in elementary torch operations or, where `own` is set, by the package's entry points.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
EPS = 1e-5                          # of the norms
LR, BETA1, BETA2, ADAM_EPS, DECAY, MAX_NORM = 3e-4, 0.9, 0.95, 1e-8, 0.1, 1.0
BLOCK = 256                         # elements that share a step of an 8-bit state
STEP0 = 1000                        # steps that went before


def listed():
    return [
        # One token's stream in front of a head: latency.
        dict(name="layernorm-fwd-1x2048", op="layernorm_fwd", rows=1, cols=2048, residual=False, beta=True, stats=False),
        # The residual stream of a GPT-2-small block (8192 tokens).
        dict(name="layernorm-fwd-8192x768", op="layernorm_fwd", rows=8192, cols=768, residual=True, beta=True, stats=True),
        # The residual stream of a LLaMA-1B-wide block (16384 tokens), the widest of the package's benchmark.
        dict(name="layernorm-fwd-16384x2048", op="layernorm_fwd", rows=16384, cols=2048, residual=True, beta=True, stats=True),
        # A short ragged batch whose rows fill no piece of a wave.
        dict(name="layernorm-bwd-257x1001", op="layernorm_bwd", rows=257, cols=1001, residual=False, beta=True),
        # 96 images of 197 tokens in a ViT-B block.
        dict(name="layernorm-bwd-18912x768", op="layernorm_bwd", rows=18912, cols=768, residual=True, beta=True),
        # The LLaMA-1B-wide stream.
        dict(name="layernorm-bwd-16384x2048", op="layernorm_bwd", rows=16384, cols=2048, residual=True, beta=True),
        # The gradients of a small model: many tensors, hardly one of a round size.
        dict(name="sumsq-ragged-61", op="sumsq", layout="ragged", tensors=61, numel=3_000_017),
        # Four LLaMA-1B blocks.
        dict(name="sumsq-llama-4", op="sumsq", layout="llama", tensors=4, numel=0),
        # A 512-wide layer, the smallest of the package's workloads, without a second copy of the weights: latency.
        dict(name="adamw32-single", op="adamw", layout="ragged", tensors=1, numel=512 * 512, bits=32, param="bf16", master=False, clip=False),
        # One LLaMA-1B block as mixed precision trains it: bf16 weights beside fp32 ones, clipped.
        dict(name="adamw32-llama-1", op="adamw", layout="llama", tensors=1, numel=0, bits=32, param="bf16", master=True, clip=True),
        # A small model with fp32 weights, many tensors of odd sizes.
        dict(name="adamw8-ragged-61", op="adamw", layout="ragged", tensors=61, numel=3_000_017, bits=8, param="fp32", master=False, clip=True),
        # Four LLaMA-1B blocks, states in 8 bits.
        dict(name="adamw8-llama-4", op="adamw", layout="llama", tensors=4, numel=0, bits=8, param="bf16", master=True, clip=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["layernorm_fwd", "layernorm_bwd", "sumsq", "adamw", "adamw"])
    if op in ("layernorm_fwd", "layernorm_bwd"):
        cols = _log_int(rng, 64, 8192)
        if rng.random() < 0.6:  # most widths are round, many are not
            cols = (cols + 15) // 16 * 16
        case = dict(op=op, rows=_log_int(rng, 1, min(65536, (1 << 25) // cols)), cols=cols, residual=rng.random() < 0.5, beta=rng.random() < 0.8)
        return {**case, "stats": rng.random() < 0.7} if op == "layernorm_fwd" else case
    llama = rng.random() < 0.2
    case = dict(op=op, layout="llama" if llama else "ragged", tensors=rng.randint(1, 2) if llama else _log_int(rng, 1, 200),
                numel=0 if llama else _log_int(rng, 20_000, 100_000_000))
    if op == "adamw":
        param = rng.choice(["bf16", "fp32"])
        case.update(bits=rng.choice([32, 8]), param=param, master=param == "bf16" and rng.random() < 0.6, clip=rng.random() < 0.7)
    return case


# ------------------------------------------------------------------------------------ inputs
def _gen(seed, index):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1009 + index) & 0x7FFFFFFFFFFF)
    return g


def _normal(shape, std, seed, index):
    return torch.randn(shape, generator=_gen(seed, index), device=DEV) * std


def _layernorm_inputs(case, seed):
    """A residual stream as an untreated model has it: a few extreme values among the ordinary ones."""
    shape = (case["rows"], case["cols"])
    x = _normal(shape, 1.0, seed, 0)
    g = _gen(seed, 50)
    at = torch.randint(0, x.numel(), (x.numel() // 10000 + 1,), generator=g, device=DEV)
    x.view(-1)[at] = 1000.0 + (at % 4000).float()
    t = dict(x=x.bfloat16(), gamma=(1 + _normal(shape[1:], 0.1, seed, 1)).bfloat16(),
             beta=_normal(shape[1:], 0.1, seed, 2).bfloat16() if case["beta"] else None,
             residual=_normal(shape, 1.0, seed, 3).bfloat16() if case["residual"] else None)
    if case["op"] == "layernorm_bwd":
        t["dy"] = _normal(shape, 1.0, seed, 4).bfloat16()
        h = t["x"].double()
        mean = h.mean(1, keepdim=True)
        t["stats"] = torch.cat([mean, 1 / ((h - mean).square().mean(1, keepdim=True) + EPS).sqrt()], 1)
    return t


def _sizes(case):
    """(elements, whether it is a matrix: only those decay and have bf16 gradients) of the tensors."""
    if case["layout"] == "llama":  # qkv, o, gate, up, down and the two norms' gains
        w = 2048
        return [(w * 3 * w, True), (w * w, True), (w * 5632, True), (w * 5632, True), (w * 5632, True), (w, False), (w, False)] * case["tensors"]
    if case["tensors"] == 1:
        return [(case["numel"], True)]
    rng = random.Random(case["tensors"] * 1000003 + case["numel"])
    share = [math.exp(rng.gauss(0, 1.0)) if i % 3 else 0.01 * rng.random() for i in range(case["tensors"])]
    return [(max(1, round(case["numel"] * s / sum(share))), i % 3 != 0) for i, s in enumerate(share)]


def _views(flat, sizes, step=1):
    """Tensors in one buffer, each on a place of its own that is a multiple of 1024 elements."""
    got, at = [], 0
    for n, _ in sizes:
        got.append(flat[at // step:at // step + -(-n // step)])
        at += -(-n // 1024) * 1024
    return got


def _flat(sizes, dtype, step=1):
    return torch.zeros(sum(-(-n // 1024) * 1024 for n, _ in sizes) // step, dtype=dtype, device=DEV)


def _model(case, seed):
    sizes = _sizes(case)
    grads = [_normal((n,), 0.01, seed, 10 + 7 * i) for i, (n, _) in enumerate(sizes)]
    s = dict(sizes=sizes, grads=[g.bfloat16() if matrix else g for g, (_, matrix) in zip(grads, sizes)])
    s["sumsq"] = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().reshape(1)
    if case["op"] == "sumsq":
        return s
    dtype, state = torch.float32 if case["param"] == "fp32" else torch.bfloat16, torch.float32 if case["bits"] == 32 else torch.uint8
    s.update(param=_flat(sizes, dtype), m=_flat(sizes, state), v=_flat(sizes, state), t=STEP0)
    if case["master"]:
        s["master"] = _flat(sizes, torch.float32)
    if case["bits"] == 8:
        s.update(m_step=_flat(sizes, torch.float32, BLOCK), v_step=_flat(sizes, torch.float32, BLOCK))
    for i, t in enumerate(_tensors(s)):
        p, m, v = (_normal(t["param"].shape, std, seed, 11 + 7 * i + j) for j, std in enumerate((0.02, 0.003, 0.01)))
        # states that many steps have left: v near the mean square of the gradients, never far below m's square
        v = v.square() * 0.5 + m.square() + 2e-5
        t["param"].copy_(p)
        if case["master"]:
            t["master"].copy_(p)
        if case["bits"] == 32:
            t["m"].copy_(m)
            t["v"].copy_(v)
            continue
        for name, x, top, kind in (("m", m, 448.0, torch.float8_e4m3fn), ("v", v, 57344.0, torch.float8_e5m2)):
            rows = _blocks(x)
            scale = top / rows.abs().amax(1, keepdim=True)
            t[name].copy_((rows * scale).clamp(-top, top).to(kind).view(torch.uint8).view(-1)[:p.numel()])
            t[name + "_step"].copy_((1 / scale).view(-1))
    return s


def _blocks(x):
    return torch.cat([x, x.new_zeros(-x.numel() % BLOCK)]).view(-1, BLOCK)


def _tensors(s):
    """The state's tensors, one dict each."""
    names = [k for k in ("param", "master", "m", "v", "m_step", "v_step") if k in s]
    views = {k: _views(s[k], s["sizes"], BLOCK if k.endswith("_step") else 1) for k in names}
    return [dict({k: views[k][i] for k in names}, grad=s["grads"][i], weight_decay=DECAY if matrix else 0.0)
            for i, (_, matrix) in enumerate(s["sizes"])]


def prepare(case, seed):
    s = dict(case=case)
    if case["op"] in ("layernorm_fwd", "layernorm_bwd"):
        s.update(_layernorm_inputs(case, seed))
        bf = lambda: torch.empty((case["rows"], case["cols"]), dtype=torch.bfloat16, device=DEV)  # noqa: E731
        f32 = lambda: torch.empty(case["cols"], dtype=torch.float32, device=DEV)  # noqa: E731
        if case["op"] == "layernorm_fwd":
            s.update(y=bf(), h=bf() if case["residual"] else None,
                     stats=torch.empty((case["rows"], 2), dtype=torch.float64, device=DEV) if case["stats"] else None)
        else:
            s.update(dx=bf(), dgamma=f32(), dbeta=f32() if case["beta"] else None)
            if own:
                import paper_2511_23225_amd as tw
                s["workspace"] = torch.empty(tw.tweo_workspace_bytes(tw.TWEO_OP_LAYERNORM_BWD, case["rows"], case["cols"], 1), dtype=torch.uint8, device=DEV)
        return s
    s.update(_model(case, seed))
    if own:
        import paper_2511_23225_amd as tw
        if case["op"] == "sumsq":  # the norm reads the gradients alone
            tensors = [dict(grad=g) for g in s["grads"]]
        else:
            tensors = _tensors(s)
        table = torch.empty(tw.tweo_optim_table_bytes(len(tensors)), dtype=torch.uint8, device=DEV)
        s["plan"] = tw.make_optim_plan([tw.optim_tensor(**t) for t in tensors], table)
        s["workspace"] = torch.empty(tw.tweo_workspace_bytes(tw.TWEO_OP_GRAD_SUMSQ, 1, 1, 1), dtype=torch.uint8, device=DEV)
        s["out"] = torch.empty(1, dtype=torch.float64, device=DEV)
    elif case["op"] == "adamw":
        s["tensors"] = _tensors(s)
    return s


# ------------------------------------------------------------------------------- the plain forms
def _plain_layernorm_fwd(s):
    h, y = s["x"], None
    if s["residual"] is not None:
        s["h"].copy_(h.float() + s["residual"].float())
        h = s["h"]
    wide = h.double()
    mean = wide.mean(1, keepdim=True)
    rstd = 1 / ((wide - mean).square().mean(1, keepdim=True) + EPS).sqrt()
    y = (h.float() - mean.float()) * rstd.float() * s["gamma"].float()
    s["y"].copy_(y if s["beta"] is None else y + s["beta"].float())
    if s["stats"] is not None:
        s["stats"].copy_(torch.cat([mean, rstd], 1))


def _plain_layernorm_bwd(s):
    rstd, dy = s["stats"][:, 1:].float(), s["dy"].float()
    xhat, w = (s["x"].float() - s["stats"][:, :1].float()) * rstd, dy * s["gamma"].float()
    dx = rstd * (w - w.mean(1, keepdim=True) - xhat * (w * xhat).mean(1, keepdim=True))
    s["dx"].copy_(dx if s["residual"] is None else dx + s["residual"].float())
    s["dgamma"].copy_((dy * xhat).sum(0))
    if s["dbeta"] is not None:
        s["dbeta"].copy_(dy.sum(0))


def _divided(top, amax):
    """top / amax, 1 where that has no use, at most the largest number."""
    scale = torch.full_like(amax, top) / torch.where(amax > 0, amax, torch.ones_like(amax))
    return torch.where(amax > 0, scale.clamp(max=torch.finfo(torch.float32).max), torch.ones_like(scale))


def _encode(x, top, bits, factor, largest, u, least):
    """Codes and steps of blocks: as an fp32 pattern the scaled value has the 8-bit format's fields in front of the
    `bits` that are cut off, and a number of so many bits (from u, 32 of them) added first decides what they round to."""
    scale = _divided(top, x.abs().amax(1, keepdim=True))
    pattern = (x.abs() * scale * factor).view(torch.int32)
    code = ((pattern + (u >> (32 - bits)).to(torch.int32)) >> bits).clamp(max=largest)
    if least:  # a positive second moment stays positive
        code = torch.where((x > 0) & (code == 0), torch.ones_like(code), code)
    return (code | ((x.view(torch.int32) >> 24) & 0x80)).to(torch.uint8), torch.ones_like(scale) / scale


def _plain_adamw(tensor, t, clip):
    p, g = tensor.get("master", tensor["param"]).float(), tensor["grad"].float()
    if clip is not None:
        g = g * clip
    n, eight = g.numel(), "m_step" in tensor
    if eight:
        m = _blocks(tensor["m"]).view(torch.float8_e4m3fn).float() * tensor["m_step"][:, None]
        v = _blocks(tensor["v"]).view(torch.float8_e5m2).float() * tensor["v_step"][:, None]
        g = _blocks(g)
    else:
        m, v = tensor["m"], tensor["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    update = m / (v.sqrt() * (1 / math.sqrt(1 - BETA2 ** t)) + ADAM_EPS)
    p = p * (1 - LR * tensor["weight_decay"]) - update.view(-1)[:n] * (LR / (1 - BETA1 ** t))
    tensor["param"].copy_(p)
    if "master" in tensor:
        tensor["master"].copy_(p)
    if not eight:
        tensor["m"].copy_(m)
        tensor["v"].copy_(v)
        return
    u = (torch.arange(m.numel(), device=DEV) * 0x6A09E667 + t * 0x9E3779B9) & 0xFFFFFFFF
    m, m_step = _encode(m, 448.0, 20, 2.0 ** -120, 0x7E, u.view(m.shape), False)
    v, v_step = _encode(v, 57344.0, 21, 2.0 ** -112, 0x7B, u.view(v.shape), True)
    tensor["m"].copy_(m.view(-1)[:n])
    tensor["v"].copy_(v.view(-1)[:n])
    tensor["m_step"].copy_(m_step.view(-1))
    tensor["v_step"].copy_(v_step.view(-1))


def _clip(sumsq):
    return (MAX_NORM / (sumsq.sqrt() + 1e-6)).clamp(max=1.0).float()


def _as_values(s):
    """What the pass has written; the codes of 8-bit states as the numbers that they are (in units of their step)."""
    out = {k: s[k] for k in ("param", "master", "m", "v", "m_step", "v_step") if k in s}
    if "m_step" in s:
        out.update(m=s["m"].view(torch.float8_e4m3fn), v=s["v"].view(torch.float8_e5m2))
    return out


def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2511_23225_amd as tw
    if c["op"] == "layernorm_fwd":
        if own:
            tw.tweo_layernorm_fwd(s["x"], s["gamma"], s["y"], beta_bf16=s["beta"], residual_bf16=s["residual"], eps=EPS,
                                  h_out_bf16=s["h"], stats_out=s["stats"])
        else:
            _plain_layernorm_fwd(s)
        return {k: s[k] for k in ("y", "h", "stats")}
    if c["op"] == "layernorm_bwd":
        if own:
            tw.tweo_layernorm_bwd(s["dy"], s["x"], s["gamma"], s["stats"], s["dx"], s["dgamma"], dbeta=s["dbeta"],
                                  residual_grad_bf16=s["residual"], workspace=s["workspace"])
        else:
            _plain_layernorm_bwd(s)
        return {k: s[k] for k in ("dx", "dgamma", "dbeta")}
    if c["op"] == "sumsq":
        if own:
            tw.tweo_grad_sumsq(s["plan"], s["out"], s["workspace"])
            return s["out"]
        return torch.stack([g.double().square().sum() for g in s["grads"]]).sum().reshape(1)
    s["t"] += 1
    if own:
        tw.tweo_adamw_step(s["plan"], lr=LR, step=s["t"], beta1=BETA1, beta2=BETA2, eps=ADAM_EPS,
                           grad_sumsq=s["sumsq"] if c["clip"] else None, max_norm=MAX_NORM)
    else:
        clip = _clip(s["sumsq"]) if c["clip"] else None
        [_plain_adamw(t, s["t"], clip) for t in s["tensors"]]
    return _as_values(s)


def work(case):
    if case["op"] in ("layernorm_fwd", "layernorm_bwd"):
        n, rows, cols, more = case["rows"] * case["cols"], case["rows"], case["cols"], 1 + case["beta"]
        if case["op"] == "layernorm_fwd":
            return dict(bytes=n * (8 if case["residual"] else 4) + 2 * cols * more + (16 * rows if case["stats"] else 0), flops=9.0 * n)
        return dict(bytes=n * (8 if case["residual"] else 6) + 2 * cols + 4 * cols * more + 16 * rows, flops=14.0 * n)
    sizes = _sizes(case)
    n, grads = sum(k for k, _ in sizes), sum(k * (2 if matrix else 4) for k, matrix in sizes)
    if case["op"] == "sumsq":
        return dict(bytes=grads + 8, flops=2.0 * n)
    weights = 10 if case["master"] else 4 if case["param"] == "bf16" else 8
    return dict(bytes=grads + n * (weights + (16 if case["bits"] == 32 else 4 + 16 / BLOCK)), flops=16.0 * n)


# -------------------------------------------------------------------------- the same in 64 bits
def _values64(codes, kind):
    return codes.view(kind).double()


def _rounded64(x, u, top, mantissa, least_exponent, steps):
    """Values with so many mantissa bits and exponents from the least on, by the fraction u in [0, 1)."""
    y = x.abs() * steps
    _, e = torch.frexp(y)
    unit = torch.exp2(torch.clamp(e.double() - 1, min=least_exponent) - mantissa)
    return torch.sign(x) * torch.minimum(torch.floor(y / unit + u) * unit, torch.full_like(y, top))


def exact(case, seed):
    if case["op"] in ("layernorm_fwd", "layernorm_bwd"):
        t = _layernorm_inputs(case, seed)
        gamma = t["gamma"].to(torch.float64)
        if case["op"] == "layernorm_fwd":
            h = t["x"].to(torch.float64) + (0 if t["residual"] is None else t["residual"].to(torch.float64))
            stored = h.to(torch.bfloat16).to(torch.float64)
            var, mean = torch.var_mean(stored, dim=1, unbiased=False, keepdim=True)
            scale = torch.rsqrt(var + EPS)
            y = (stored - mean) * scale * gamma + (0 if t["beta"] is None else t["beta"].to(torch.float64))
            return dict(y=y, h=None if t["residual"] is None else h, stats=torch.hstack([mean, scale]) if case["stats"] else None)
        x, dy = t["x"].to(torch.float64).requires_grad_(), t["dy"].to(torch.float64)
        gamma.requires_grad_()
        # the norm's own formula, differentiated
        xhat = (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + EPS).sqrt()
        dx, dgamma = torch.autograd.grad((xhat * gamma * dy).sum(), (x, gamma))
        return dict(dx=dx if t["residual"] is None else dx + t["residual"].to(torch.float64), dgamma=dgamma, dbeta=dy.sum(0) if case["beta"] else None)
    s = _model(case, seed)
    total = sum(float(torch.dot(g.double(), g.double())) for g in s["grads"])
    if case["op"] == "sumsq":
        return torch.tensor([total], dtype=torch.float64, device=DEV)
    clip = min(1.0, MAX_NORM / (math.sqrt(total) + 1e-6)) if case["clip"] else 1.0
    out = {k: torch.zeros(s[k].numel(), dtype=torch.float64, device=DEV) for k in ("param", "master", "m", "v", "m_step", "v_step") if k in s}
    at, t = 0, STEP0 + 1
    for i, (n, matrix) in enumerate(s["sizes"]):
        here, blocks = slice(at, at + n), slice(at // BLOCK, at // BLOCK + -(-n // BLOCK))
        at += -(-n // 1024) * 1024
        g, p = s["grads"][i].double() * clip, s["master" if case["master"] else "param"][here].double()
        m, v = s["m"][here], s["v"][here]
        if case["bits"] == 8:
            block = torch.arange(n, device=DEV) // BLOCK
            m = _values64(m, torch.float8_e4m3fn) * s["m_step"][blocks].double()[block]
            v = _values64(v, torch.float8_e5m2) * s["v_step"][blocks].double()[block]
        m = BETA1 * m.double() + (1 - BETA1) * g
        v = BETA2 * v.double() + (1 - BETA2) * g ** 2
        p = p - LR * (DECAY if matrix else 0.0) * p - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + ADAM_EPS)
        out["param"][here] = p
        if case["master"]:
            out["master"][here] = p
        if case["bits"] == 8:
            w = torch.remainder(torch.arange(n, device=DEV) * 0x6A09E667 + t * 0x9E3779B9, 2 ** 32)
            for name, x, top, mantissa, least in (("m", m, 448.0, 3, -6), ("v", v, 57344.0, 2, -14)):
                amax = torch.zeros(blocks.stop - blocks.start, dtype=torch.float64, device=DEV).scatter_reduce_(0, block, x.abs(), "amax")
                scale = torch.where(amax > 0, top / amax, torch.ones_like(amax))
                u = torch.floor(w / 2 ** (9 + mantissa)) / 2 ** (23 - mantissa)
                q = _rounded64(x, u, top, mantissa, least, scale[block])
                if name == "v":
                    q = torch.where((x > 0) & (q == 0), torch.full_like(q, 2.0 ** -16), q)
                out[name][here], out[name + "_step"][blocks] = q, 1 / scale
        else:
            out["m"][here], out["v"][here] = m, v
    return out
