"""Registers of the kernels of a mixture-of-experts layer in training, from the compiler's own metadata (no GPU): two waves of a tile kernel
share a SIMD, the few-row kernel's have one each, the row kernels' leave room for seven or eight, and nothing goes through scratch memory."""
import re
from concurrent.futures import ThreadPoolExecutor

from tests.test_register_budget import kernel_registers


def test_moe_train_kernels():
    with ThreadPoolExecutor(2) as ex:
        parts = list(ex.map(kernel_registers, ["tl_moe_rows.hip", "tl_moe_products.hip"]))
    regs = {k: v for part in parts for k, v in part.items()}
    for name, most in (("moe_product_kernel", 256), ("moe_grad_w_kernel", 256), ("moe_grad_w_join_kernel", 128), ("moe_grad_w_plan_kernel", 64), ("moe_few_rows_kernel", 512),
                       ("moe_dispatch_kernel", 64), ("moe_gather_sum_kernel", 64), ("moe_combine_grad_kernel", 72), ("moe_route_grad_kernel", 64),
                       ("moe_place_kernel", 64), ("moe_count_kernel", 64)):
        hits = [k for k in regs if re.search(name, k)]
        assert hits, name
        for k in hits:
            assert regs[k]["vgpr"] <= most, (k, regs[k])
    for k, r in regs.items():
        assert r["spill"] == 0 and r["scratch"] == 0, (k, r)
