"""Without a GPU: what the gated feed-forward's entry points refuse before anything is launched, and pins of the oracle."""
import ctypes

import numpy as np
import pytest

import paper_2511_23225_amd as tw
from oracle import block


@pytest.fixture(scope="module")
def memory():
    """Addresses of host memory, 256-byte aligned, 64 KB apart; nothing reads them."""
    buf = ctypes.create_string_buffer(1 << 21)
    first = (ctypes.addressof(buf) + 255) & ~255
    yield [first + i * 65536 for i in range(24)]
    del buf


def test_forward_refusals(memory):
    xq, sx, wq, sw, h, gu = memory[:6]
    lib = tw.load()
    good = dict(xq=xq, sx=sx, wq=wq, sw=sw, M=16, F=24, K=32, act=0, h=h, gu=gu)

    def fwd(**k):
        a = {**good, **k}
        return lib.tweo_fp8_gated_fwd(a["xq"], a["sx"], a["wq"], a["sw"], a["M"], a["F"], a["K"], a["act"], a["h"], a["gu"], None)

    for k in (dict(xq=None), dict(sx=None), dict(wq=None), dict(sw=None), dict(h=None), dict(xq=xq + 8), dict(wq=wq + 4), dict(h=h + 2), dict(gu=gu + 8),
              dict(sx=sx + 2), dict(M=0), dict(F=0), dict(K=0), dict(M=-1), dict(F=-8), dict(act=2), dict(act=-1), dict(h=gu), dict(h=gu + 16), dict(h=xq),
              dict(gu=wq), dict(gu=sx), dict(h=h, gu=h + 16 * 24 * 2 - 16)):
        assert fwd(**k) == tw.TWEO_ERR_INVALID_ARG, k
    for k in (dict(F=20), dict(K=24), dict(M=(1 << 30) + 1), dict(F=(1 << 24) + 8), dict(F=1 << 24), dict(K=(1 << 24) + 16), dict(M=1 << 30, F=1 << 20)):
        assert fwd(**k) == tw.TWEO_ERR_UNSUPPORTED, k


def test_w8a8_refusals(memory):
    xq, wq, xs, ws, h = memory[:5]
    lib = tw.load()
    good = dict(xq=xq, wq=wq, M=16, F=24, K=32, xs=xs, xt=1, ws=ws, wc=1, act=0, h=h, inv=1.0)

    def both(**k):
        a = {**good, **k}
        head = a["xq"], a["wq"], a["M"], a["F"], a["K"], a["xs"], a["xt"], a["ws"], a["wc"], a["act"]
        got = {lib.tweo_w8a8_gated_i8out(*head, a["inv"], a["h"], None)}
        if "inv" not in k:
            got.add(lib.tweo_w8a8_gated(*head, a["h"], None))
        return got

    for k in (dict(xq=None), dict(wq=None), dict(xs=None), dict(ws=None), dict(h=None), dict(xq=xq + 8), dict(wq=wq + 1), dict(h=h + 8), dict(xs=xs + 2),
              dict(ws=ws + 1), dict(xt=2), dict(wc=-1), dict(M=0), dict(F=0), dict(K=0), dict(act=2), dict(h=xq), dict(h=wq + 16), dict(h=ws), dict(h=xs),
              dict(inv=float("nan"))):
        assert both(**k) == {tw.TWEO_ERR_INVALID_ARG}, k
    for k in (dict(F=20), dict(K=40), dict(M=(1 << 30) + 1), dict(F=1 << 24)):
        assert both(**k) == {tw.TWEO_ERR_UNSUPPORTED}, k


def test_whole_path_refusals(memory):
    names = ("x", "w", "h", "gu", "xq", "xqT", "wq", "wqT", "sc", "stx", "stw", "ws", "dh", "q", "qT", "dx", "dw", "std")
    base = dict(zip(names, memory))
    lib = tw.load()
    base.update(M=16, F=24, K=32, act=0, n=1 << 16, e5m2=0)

    def saved(a):
        return None if a.get("saved", 0) is None else ctypes.byref(tw.binding.Fp8Saved(a["xq"], a["xqT"], a["wq"], a["wqT"], a["sc"]))

    def fwd(**k):
        a = {**base, "stx": None, "stw": None, **k}
        return lib.tweo_fp8_gated_fwd_bf16(a["x"], a["w"], a["M"], a["F"], a["K"], a["act"], a["h"], a["gu"], saved(a), a["stx"], a["stw"], 0, a["ws"], a["n"],
                                           None)

    for k in (dict(x=None), dict(w=None), dict(h=None), dict(saved=None), dict(xq=None), dict(xqT=None), dict(wq=None), dict(wqT=None), dict(sc=None),
              dict(x=base["x"] + 2), dict(w=base["w"] + 8), dict(h=base["h"] + 2), dict(gu=base["gu"] + 2), dict(xqT=base["xqT"] + 8), dict(act=3), dict(M=0),
              dict(stx=base["stx"]), dict(stw=base["stw"]), dict(stx=base["stx"], stw=base["stx"]), dict(stx=base["stx"] + 4, stw=base["stw"]),
              dict(h=base["x"]), dict(gu=base["h"]), dict(xq=base["xqT"]), dict(ws=base["h"]), dict(sc=base["ws"]), dict(stx=base["sc"], stw=base["stw"])):
        assert fwd(**k) == tw.TWEO_ERR_INVALID_ARG, k
    for k in (dict(M=17), dict(F=20), dict(K=40)):
        assert fwd(**k) == tw.TWEO_ERR_UNSUPPORTED, k
    for k in (dict(ws=None), dict(ws=base["ws"] + 8), dict(n=4095)):
        assert fwd(**k) == tw.TWEO_ERR_WORKSPACE, k

    def bwd(**k):
        a = {**base, "std": None, **k}
        return lib.tweo_fp8_gated_bwd_bf16(a["dh"], a["gu"], saved(a), a["M"], a["F"], a["K"], a["act"], a["e5m2"], a["std"], 0, a["q"], a["qT"], a["dx"],
                                           a["dw"], a["ws"], a["n"], None)

    for k in (dict(dh=None), dict(gu=None), dict(saved=None), dict(xqT=None), dict(wqT=None), dict(sc=None), dict(q=None), dict(qT=None),
              dict(dh=base["dh"] + 2), dict(gu=base["gu"] + 8), dict(q=base["q"] + 8), dict(qT=base["qT"] + 1), dict(dx=base["dx"] + 2), dict(dw=base["dw"] + 2),
              dict(e5m2=2), dict(act=2), dict(std=base["std"] + 4), dict(F=0), dict(q=base["dh"]), dict(dx=base["gu"]), dict(dw=base["wqT"]), dict(qT=base["q"]),
              dict(ws=base["dx"]), dict(std=base["sc"])):
        assert bwd(**k) == tw.TWEO_ERR_INVALID_ARG, k
    for k in (dict(M=24), dict(F=12), dict(K=8)):
        assert bwd(**k) == tw.TWEO_ERR_UNSUPPORTED, k
    for k in (dict(ws=None), dict(ws=base["ws"] + 8), dict(n=4095)):
        assert bwd(**k) == tw.TWEO_ERR_WORKSPACE, k
    for op in (tw.TWEO_OP_FP8_GATED_FWD_BF16, tw.TWEO_OP_FP8_GATED_BWD_BF16):
        b = tw.tweo_workspace_bytes(op, 16384, 5632, 2048)
        assert b >= 4096 and b % 256 == 0
    assert tw.tweo_workspace_bytes(tw.TWEO_OP_FP8_GATED_BWD_BF16, 8192, 2304, 768) == 4096 + tw.tweo_workspace_bytes(tw.TWEO_OP_FP8_LINEAR_BWD, 8192, 4608, 768)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_oracle_activation(act):
    g = np.concatenate([np.linspace(-12, 12, 97), [0.0]])
    a = block.activation(g, act)
    assert a[-1] == 0 and np.allclose(a[48], 0) and np.allclose(block.activation(np.array([30.0]), act), 30.0) and abs(block.activation(np.array([-30.0]), act)) < 1e-10
    h = 1e-5
    assert np.allclose((block.activation(g + h, act) - block.activation(g - h, act)) / (2 * h), block.activation_slope(g, act), rtol=1e-7, atol=1e-9)
    if act == "gelu":  # the tanh form, near the error function's
        t = 0.5 * g * (1 + np.tanh(block.GELU[0] * (g + block.GELU[1] * g ** 3)))
        assert np.allclose(t, a, rtol=1e-12, atol=1e-15)
        from math import erf
        assert np.abs(a - np.array([v * 0.5 * (1 + erf(v / 2 ** 0.5)) for v in g])).max() < 5e-4
