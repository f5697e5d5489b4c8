"""Without a GPU: calls of the norm and optimizer entry points that would read or write the wrong memory, or count it wrongly, are refused
before anything is launched."""
import ctypes
import os
import re

import pytest
import torch

import paper_2511_23225_amd as tw


@pytest.fixture(scope="module")
def lib():
    return tw.load()


@pytest.fixture(scope="module")
def memory():
    """Addresses of host memory, 256-byte aligned, 64 KB apart; nothing reads them."""
    buf = ctypes.create_string_buffer(1 << 21)
    first = (ctypes.addressof(buf) + 255) & ~255
    yield [first + i * 65536 for i in range(24)]
    del buf


def test_workspace_of_a_backward_pass_of_few_rows(lib):
    """Its one launch leaves nothing in it."""
    need = lambda rows, cols: tw.tweo_workspace_bytes(tw.TWEO_OP_LAYERNORM_BWD, rows, cols, 1)  # noqa: E731
    for rows, cols in ((1, 1), (4, 16), (512, 8192), (300, 768)):
        assert need(rows, cols) == 256, (rows, cols)
    # of more, a row of partial sums of both gradients a workgroup
    assert need(513, 8192) >= 256 * 2 * 8192 * 4 and need(512, 8200) >= 2 * 8200 * 4 and need(513, 64) >= 2 * 64 * 4


def test_layernorm_buffers_that_overlap(lib, memory):
    """What a call writes may be one of the tensors that the header names, exactly, and touches nothing else that the call reads or writes.
    The statistics in the backward pass's own workspace among them: its partial sums would go over them while they are read."""
    x, r, g, b, h, y, st, far = memory[:8]
    size = 4 * 16 * 2
    good = dict(x=x, r=r, g=g, b=b, rows=4, cols=16, h=h, y=y, st=st)

    def fwd(**k):
        a = {**good, **k}
        return lib.tweo_layernorm_fwd(a["x"], a["r"], a["g"], a["b"], a["rows"], a["cols"], 1e-5, a["h"], a["y"], a["st"], None)

    bad = [dict(y=x + 16), dict(y=x - size + 16), dict(y=r + 32), dict(h=x + 16), dict(h=r - 16), dict(h=y), dict(h=y + 16), dict(y=h - 16), dict(y=g), dict(y=b),
           dict(h=g - size + 16), dict(st=x), dict(st=r + 16), dict(st=y + size - 16), dict(st=h), dict(st=g), dict(st=b + 16),
           dict(h=x, y=x), dict(h=r, y=r), dict(r=x, h=x, y=x), dict(r=None, y=x + 16), dict(r=None, y=x, st=x), dict(r=None, y=g)]
    for k in bad:
        assert fwd(**k) == tw.TWEO_ERR_INVALID_ARG, k
    good = dict(dy=x, h=h, g=g, st=st, dres=r, rows=600, cols=16, dx=y, dg=b, db=b + 64, ws=far, n=1 << 15)
    size = 600 * 16 * 2

    def bwd(**k):
        a = {**good, **k}
        return lib.tweo_layernorm_bwd(a["dy"], a["h"], a["g"], a["st"], a["dres"], a["rows"], a["cols"], a["dx"], a["dg"], a["db"], a["ws"], a["n"], None)

    need = tw.tweo_workspace_bytes(tw.TWEO_OP_LAYERNORM_BWD, 600, 16, 1)
    assert 256 < need < 1 << 15
    bad = [dict(st=far), dict(st=far + 256), dict(st=far + 2304), dict(st=far - 600 * 16 + 16), dict(h=far), dict(dx=far), dict(dg=far), dict(g=far + 16),
           dict(dx=h), dict(dx=h + 16), dict(dx=x + 16), dict(dx=r - 16), dict(dx=st), dict(dx=g), dict(dg=b + 16, db=b), dict(db=b), dict(dg=h + size - 16),
           dict(db=st), dict(dg=g), dict(dg=y), dict(db=x), dict(dy=h, dx=h), dict(dres=h, dx=h)]
    for k in bad:
        assert bwd(**k) == tw.TWEO_ERR_INVALID_ARG, k
    # few rows in one launch: other workgroups read h while dx is written
    for k in (dict(dx=h), dict(dx=h + 16), dict(dx=st), dict(dg=b, db=b)):
        assert bwd(rows=12, **k) == tw.TWEO_ERR_INVALID_ARG, k


def test_an_eps_without_a_reciprocal(lib, memory):
    """Below 2^-126 1 / eps is beyond fp32 (or eps is 0 there), and 0 times it would make NaN of a parameter whose gradients have been zero."""
    plan = tw.binding.OptimPlan(memory[0], 4, 1, 32)
    for eps in (1e-40, 1e-60, 5e-324, 2.0 ** -127, 2.0 ** -126 * (1 - 2.0 ** -23)):
        cfg = tw.binding.AdamwCfg(1e-3, 0.9, 0.999, eps, 1.0, 1)
        assert lib.tweo_adamw_step(ctypes.byref(plan), ctypes.byref(cfg), None, None, None) == tw.TWEO_ERR_INVALID_ARG, eps


class Elsewhere:
    """A tensor that says it is on the device it is asked for, for checks that come before any launch."""

    def __init__(self, t, device=0):
        self.t, self.device = t, device

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.device


@pytest.fixture
def on_device(monkeypatch):
    """A current device without a GPU, and entry points that note that they were reached."""
    reached = []

    class Reached:
        def __getattr__(self, name):
            return lambda *a: reached.append(name) or tw.TWEO_OK

    monkeypatch.setattr(tw.binding, "_current", (lambda: 0, lambda device: None))
    monkeypatch.setattr(tw.binding, "_lib", Reached())
    plan = tw.binding.OptimPlan()
    plan.device = 0
    return plan, reached


def test_a_schedule_is_two_integer_words(on_device):
    plan, reached = on_device
    words = torch.zeros(8, dtype=torch.int32)
    for bad in (torch.tensor([1e-3, 1000.0]), torch.zeros(2, dtype=torch.int64), torch.zeros(4, dtype=torch.int16), torch.zeros(2, dtype=torch.float64),
                words[::2], words[:1], torch.zeros(1, dtype=torch.int32).expand(2)):
        with pytest.raises(ValueError):
            tw.tweo_adamw_step(plan, schedule=Elsewhere(bad))
    with pytest.raises(ValueError):
        tw.tweo_adamw_step(plan, schedule=Elsewhere(words[:2], -1))
    assert not reached
    tw.tweo_adamw_step(plan, schedule=Elsewhere(words[:2]))
    tw.tweo_adamw_step(plan, schedule=Elsewhere(words[4:].view(torch.uint32)))
    assert reached == ["tweo_adamw_step"] * 2


def test_statistics_in_a_workspace_of_any_type():
    """The offset is in bytes, whatever the workspace's type; what is too short, or does not lie in one piece, is refused."""
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "tweo.h")).read()
    assert int(re.search(r"#define TWEO_LAYERNORM_STATS_OFFSET (\d+)", header).group(1)) == tw.binding.LAYERNORM_STATS_OFFSET
    rows, offset = 48, tw.binding.LAYERNORM_STATS_OFFSET
    need = tw.tweo_workspace_bytes(tw.TWEO_OP_LAYERNORM_QUANTIZE, rows, 1, 1)
    whole = torch.zeros(need + 64, dtype=torch.uint8)
    want = torch.arange(2 * rows, dtype=torch.float64)
    whole[offset:offset + 16 * rows] = want.view(torch.uint8)
    for kind in (torch.uint8, torch.int8, torch.int32, torch.float32, torch.float64, torch.bfloat16):
        got = tw.layernorm_stats(whole[:need].view(kind), rows)
        assert torch.equal(got, want.view(rows, 2)) and got.data_ptr() == whole.data_ptr() + offset, kind
    assert torch.equal(tw.layernorm_stats(whole[:need].view(4, -1), rows), want.view(rows, 2))
    for bad, count in ((whole[:need:2], rows), (whole[:offset + 16 * rows - 1], rows), (whole[:offset], 1), (whole, 0), (whole, -1), (whole[:need], 1 << 20)):
        with pytest.raises(ValueError):
            tw.layernorm_stats(bad, count)


def test_scratch_memory_lies_in_one_piece(on_device):
    """The library takes an address and a number of bytes: of a tensor with strides they would name memory that is not its own."""
    plan, reached = on_device
    n = 1 << 16
    for bad in (Elsewhere(torch.zeros(2 * n, dtype=torch.uint8)[::2]), Elsewhere(torch.zeros(1, dtype=torch.uint8).expand(n)),
                Elsewhere(torch.zeros((64, n // 32), dtype=torch.uint8)[:, :n // 64]), Elsewhere(torch.zeros(n, dtype=torch.uint8), 1)):
        with pytest.raises(ValueError):
            tw.tweo_grad_sumsq(plan, Elsewhere(torch.zeros(1, dtype=torch.float64)), bad)
        with pytest.raises(ValueError):
            tw.make_optim_plan([], bad)
        x, row = Elsewhere(torch.zeros((4, 16), dtype=torch.bfloat16)), Elsewhere(torch.zeros(16, dtype=torch.bfloat16))
        with pytest.raises(ValueError):
            tw.tweo_layernorm_bwd(x, x, row, Elsewhere(torch.zeros((4, 2), dtype=torch.float64)), x, Elsewhere(torch.zeros(16)), workspace=bad)
    assert not reached
    good = Elsewhere(torch.zeros(n, dtype=torch.uint8))
    tw.tweo_grad_sumsq(plan, Elsewhere(torch.zeros(1, dtype=torch.float64)), good)
    tw.make_optim_plan([], good)
    assert reached == ["tweo_grad_sumsq", "tweo_optim_plan_init"]
