"""Registers of the paged-cache kernels, from the compiler's own metadata (no GPU): two waves of the attention kernels share a SIMD
(8 waves a workgroup, one workgroup a compute unit), and nothing goes through scratch memory, whose accesses would wait for
the block loads in flight."""
import re
from concurrent.futures import ThreadPoolExecutor

from tests.test_register_budget import kernel_registers


def test_paged_kernels():
    with ThreadPoolExecutor(2) as ex:
        parts = list(ex.map(kernel_registers, ["tl_paged.hip", "tl_qk_norm_rope.hip"]))
    regs = {k: v for part in parts for k, v in part.items()}
    for name, most in (("paged_mixed_kernel", 256), ("paged_few_rows_kernel", 256), ("paged_join_kernel", 64), ("paged_schedule_kernel", 128),
                       ("paged_slots_kernel", 128), ("qk_norm_rope_kernel", 64)):
        hits = [k for k in regs if re.search(name, k)]
        assert hits, name
        for k in hits:
            assert regs[k]["vgpr"] <= most, (k, regs[k])
    for k, r in regs.items():
        assert r["spill"] == 0 and r["scratch"] == 0, (k, r)
