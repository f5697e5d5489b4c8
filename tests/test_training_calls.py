"""Without a GPU: calls of the norm and optimizer entry points that would read or write the wrong memory, or count it wrongly, are refused
before anything is launched."""
import ctypes

import pytest

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
