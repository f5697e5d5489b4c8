"""Sizes at the ends of what the entry points on heads take, as include/tweo.h states them (no GPU needed): one more is refused as unsupported; at the
end itself the call gets to its buffers, which overlap here, so that nothing is launched."""
import ctypes

import pytest

import paper_2511_23225_amd as tw

LIMIT = 1 << 46


@pytest.fixture(scope="module")
def memory():
    """An address that nothing reads."""
    buf = ctypes.create_string_buffer(4096)
    yield (ctypes.addressof(buf) + 255) & ~255
    del buf


def calls(at, tokens, heads, token=64, head=64, dim=16):
    """What each entry point says to heads whose input begins in the middle of the output's first."""
    row = tw.binding.Heads(at, at + 2, token, head, token, head, None, heads)
    grad = tw.binding.HeadsGrad(at, at, at + 2, token, head, token, head, token, head, None, None, heads)
    cfg = ctypes.byref(tw.binding.RotaryCfg(at + 1024, at + 2048, 2, 0, 1.0))
    lib = tw.load()
    return {lib.tweo_rotary(ctypes.byref(row), 1, tokens, dim, cfg, 0, None), lib.tweo_head_norm_rotary_fwd(ctypes.byref(row), 1, tokens, dim, 1e-6, cfg, None),
            lib.tweo_head_norm_rotary_bwd(ctypes.byref(grad), 1, tokens, dim, 1e-6, cfg, None, 0, None)}


@pytest.mark.parametrize("at_end,beyond", [
    (dict(tokens=1 << 30, heads=16), dict(tokens=(1 << 30) + 1, heads=1)),
    (dict(tokens=1 << 18, heads=1 << 16), dict(tokens=(1 << 18) + 1, heads=1 << 16)),
    (dict(tokens=1, heads=1 << 16), dict(tokens=1, heads=(1 << 16) + 1)),
    (dict(tokens=1, heads=1, dim=512), dict(tokens=1, heads=1, dim=513)),
    (dict(tokens=4, heads=1, token=LIMIT // 4), dict(tokens=4, heads=1, token=LIMIT // 4 + 1)),
    (dict(tokens=1, heads=4, head=LIMIT // 4), dict(tokens=1, heads=4, head=LIMIT // 4 + 1)),
])
def test_ends(memory, at_end, beyond):
    assert calls(memory, **at_end) == {tw.TWEO_ERR_INVALID_ARG}
    assert calls(memory, **beyond) == {tw.TWEO_ERR_UNSUPPORTED}


def test_strides_that_nothing_is_reached_by(memory):
    far = (1 << 63) - 1
    assert calls(memory, tokens=1, heads=1, token=far, head=far) == {tw.TWEO_ERR_INVALID_ARG}
    assert calls(memory, tokens=1, heads=1, token=-1) == {tw.TWEO_ERR_INVALID_ARG}
