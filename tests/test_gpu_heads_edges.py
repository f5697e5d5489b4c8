"""Rotary positions and head norms at the ends of what they take, on the GPU, against fp64.  Bounds of single results as in test_gpu_heads.py."""
import numpy as np
import pytest
import torch

import paper_2511_23225_amd as tw
from oracle import block
from gpu_util import DEV
from test_gpu_heads import EPS, U, bf, f64, freqs_of, near

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
