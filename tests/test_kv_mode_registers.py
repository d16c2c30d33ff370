"""The attention kernels' other modes keep their sums in ordinary registers too (test_kv_registers.py says why)."""
from test_kv_registers import kernels  # noqa: F401


def test_no_kernel_of_a_mode_uses_accumulation_registers(kernels):  # noqa: F811
    modes = {n: k for n, k in kernels.items() if "kv_few_mode_kernel" in n or "kv_many_mode_kernel" in n}
    # first tokens beside a window, and lists: each as many instances as the plain kernels
    assert len(modes) == 2 * (14 * 4 + 7)
    # both lists in one launch: wherever a 16-bit call has tiles of 32 rows
    pairs = {n: k for n, k in kernels.items() if "kv_pair_kernel" in n}
    assert len(pairs) == 7
    for name, k in {**modes, **pairs}.items():
        assert k[".agpr_count"] == 0, name
        assert k[".vgpr_count"] <= 256, name
