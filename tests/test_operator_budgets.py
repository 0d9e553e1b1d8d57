"""Registers of the operators around the expert GEMMs, from the metadata of the built code objects: none in memory.  (The norm's
gradients of rows of more than 32 KiB held in registers took 360 us where reading the row again takes 134.)"""
import re

from test_kernel_budgets import table  # noqa: F401


def test_operators_do_not_spill(table):  # noqa: F811
    found = {n: k for n, k in table.items() if re.search(r"rmsnorm|combine_rows|dispatch_gather|adamw", n)}
    for part in ("rmsnorm_kernel", "rmsnorm_backward_kernel", "combine_rows_kernel", "combine_rows_backward_kernel", "adamw_kernel"):
        assert sum(part in n for n in found) >= 2, part
    for n, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".sgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n
        # a SIMD's 512 registers for the waves that a workgroup has on it
        waves = max(1, k[".max_flat_workgroup_size"] // 256)
        assert k[".vgpr_count"] <= 512 // waves, (n, k[".vgpr_count"])
