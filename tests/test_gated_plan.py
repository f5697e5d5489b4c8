"""Which kernel the gated feed-forward's product runs on (no GPU needed: 256 CUs are assumed)."""
import ctypes

import pytest

import paper_2511_23225_amd as tw
import test_gpu_gated

OP = tw.TWEO_OP_FP8_GATED_FWD_BF16


def cases_of(test):
    """Variants and sizes that a test is given."""
    test = getattr(test_gpu_gated, test)
    (mark,) = [m for m in test.pytestmark if m.name == "parametrize" and m.args[0].startswith("variant")]
    for variant, *sizes in mark.args[1]:
        yield variant, sizes[0] if len(sizes) == 1 else tuple(sizes)


@pytest.mark.parametrize("test", ["test_fp8_forward_on", "test_fp8_outputs_beyond_32_bits"])
def test_forced_kernels_run(test):
    """The products that are compared with fp64 on a kernel by its number run on that kernel."""
    cases = list(cases_of(test))
    assert cases
    for variant, sizes in cases:
        for keep in (False, True):
            tw.tweo_set_gemm_tile(variant)
            try:
                assert tw.tweo_gemm_plan(OP, *sizes, residual=keep) == (variant, 1, False), (variant, sizes)
            finally:
                tw.tweo_set_gemm_tile(0)


def test_kernels_by_the_sizes():
    """By the estimated times: one token, a layer in training, rows that are no whole tiles; and where a forced kernel does not take the sizes, what is chosen without."""
    plan = lambda *sizes, **k: tw.tweo_gemm_plan(OP, *sizes, **k)[0]  # noqa: E731
    assert plan(1, 5632, 2048) == 18 and plan(16384, 5632, 2048) == 15 and plan(16384, 5632, 2048, residual=True) == 15
    assert plan(1395, 9248, 3616) == 24 and plan(926, 7680, 256) == 21 and plan(768, 9728, 5632) == 15
    for variant, sizes in ((15, (300, 1000, 2048)), (15, (256, 128, 640)), (24, (300, 1000, 896)), (22, (300, 1000, 896)), (11, (512, 512, 512))):
        tw.tweo_set_gemm_tile(variant)
        try:
            forced = plan(*sizes)
        finally:
            tw.tweo_set_gemm_tile(0)
        assert forced == plan(*sizes) != variant
    info = tw.binding.GemmPlan()
    call = lambda M, N, K: tw.load().tweo_gemm_plan(OP, M, N, K, 0, 0, 0, ctypes.byref(info))  # noqa: E731
    assert call(0, 8, 16) == tw.TWEO_ERR_INVALID_ARG and call(16, 1 << 24, 16) == tw.TWEO_ERR_UNSUPPORTED
