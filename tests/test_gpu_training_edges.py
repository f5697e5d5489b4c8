"""Norm gradients and AdamW where fp32 runs out: constant rows, values near bf16's largest, rows of a million columns, gradients whose
squares have no place in fp32."""
import numpy as np
import pytest
import torch

import paper_2511_23225_amd as tw
from oracle import training
from paper_2511_23225_amd import synth
from gpu_util import DEV, bf16_bits, to_dev_bf16, workspace
from test_gpu_layernorm_grad import EPS, backward, check_backward, f64, forward, inputs, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [3, 48, 61, 100, 121, 250, 256, 777, 768, 1000, 1001, 2041, 2048, 4093, 8191, 16392, 33001])
@pytest.mark.parametrize("rows", [10, 523])
def test_backward_of_rows_of_one_value(rows, cols):
    """Variance 0, also of values whose product with 1 / sqrt(eps) has no place in fp32: xhat is 0, so that dx is rstd (w - mean w) and
    dgamma 0, for widths that fill their pieces and for those that do not."""
    say("rows of one value", rows, cols)
    values = np.float32([5.5, -0.1, 3e38, 1e-39, 1 / 3, 0.0, 7.0, -1e30, 1.5e36, -3e38])
    t = inputs(rows, cols, 31)
    t["x"] = synth.f32_to_bf16_bits(np.repeat(np.resize(values, rows)[:, None], cols, 1))
    _, _, st = forward(t, cols, False, True)
    for residual in (False, True):
        got = backward(t, to_dev_bf16(t["x"]), st, residual)
        assert bool(torch.isfinite(got[0].float()).all()) and not bool(got[1].any())
        check_backward(t, t["x"], st.cpu().numpy(), got, residual)
