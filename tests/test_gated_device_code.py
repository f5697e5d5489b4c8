"""What the compiler made of the gated feed-forward's kernels (no GPU needed)."""
from test_device_code import code_objects, instructions  # noqa: F401


# as beside the deferred-epilogue kernel's other forms: a FLAT access may end out of order and counts in both wait counters
def test_no_flat_access_beside_counted_waits(code_objects):  # noqa: F811
    for kernel in ("gemm_nt_defer_gated_kernel", "gemm_nt_ring_gated_kernel"):
        found = instructions(code_objects, kernel)
        assert found and all("s_endpgm" in ops for ops in found.values())
        flat = {name: sum(op.startswith("flat_") for op in ops) for name, ops in found.items()}
        assert not any(flat.values()), flat
