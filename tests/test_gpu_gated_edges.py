"""The gated feed-forward's entry points at the ends of what they take, on the GPU."""
import numpy as np
import pytest
import torch

import paper_2511_23225_amd as tw
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
