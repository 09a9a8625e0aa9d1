"""Which kernel a call of a mixture-of-experts layer in training takes (no GPU): the library's own rules, built for the host alone
(host_moe_choice.hip), on the cases of the GPU tests.  A case that names its kernel takes it, and every kernel there is has a case."""
import os
import subprocess

import pytest

from tests import test_gpu_moe_products_kernels as products
from tests import test_gpu_moe_route_grad_masks as route
from tests import test_gpu_moe_rows_streaming as rows
from tests import test_gpu_moe_sort as sort

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2503_20313_amd")
HIPCC = "/opt/rocm/bin/hipcc"


@pytest.fixture(scope="module")
def kernels_of(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("choice") / "host_moe_choice")
    subprocess.run([HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"),
                    os.path.join(ROOT, "tests", "host_moe_choice.hip"), "-o", exe, "-L", PKG, "-ltilelink_mi355", f"-Wl,-rpath,{PKG}"],
                   check=True, capture_output=True, timeout=300)

    def run(calls):
        r = subprocess.run([exe], input="".join(" ".join(map(str, c)) + "\n" for c in calls), capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        return r.stdout.splitlines()
    return run


pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs the ROCm compiler")


def test_products(kernels_of):
    cases = [(kernel, products.room(counts), K, N, len(counts)) for kernel, counts, K, N in products.PRODUCTS + products.GRADIENTS_OF_WEIGHTS]
    got = kernels_of([(kernel.split()[0], *sizes) for kernel, *sizes in cases])
    assert got == [c[0] for c in cases]
    few = [f"few {s}" for s in ("wide 1 2", "wide 2 1", "narrow 2 1", "narrow 4 1")]
    tiles = [f"tiles {t} {c}" for t in (128, 256) for c in ("whole", "cut")]
    assert set(got) == {f"{op} {k}" for op in ("gemm", "gemm_grad_x") for k in few + tiles} | {f"gemm_grad_w {t} {c}" for t in ("128x128", "128x256", "256x256") for c in ("whole", "cut")}
    roomy = kernels_of([(kernel.split()[0], room, K, N, len(counts)) for kernel, counts, K, N, room in products.ROOMY])
    assert roomy == [c[0] for c in products.ROOMY]


def test_rows(kernels_of):
    cases = rows.FORWARD + rows.SUMS + rows.GRADIENTS
    got = kernels_of([(variant.split()[0], *sizes) for variant, *sizes in cases])
    assert got == [c[0] for c in cases]
    loads = ("cached", "stream")
    assert set(got) == ({f"dispatch cached {s}" for s in loads} | {f"{op} {l} cached" for op in ("dispatch_grad", "combine") for l in loads} |
                        {f"combine_grad {w} {s}" for w in (1, 4) for s in ("cached cached", "cached stream", "stream stream")})


def test_routing_weights(kernels_of):
    got = kernels_of([("route_grad", E, k) for _, _, E, k in route.SHAPES])
    assert got == ["route_grad " + s[0] for s in route.SHAPES]
    assert set(got) == {f"route_grad {lanes} {per}" for lanes in (16, 32) for per in (1, 2, 4, 8, 16) if lanes * per <= 256}


def test_sort(kernels_of):
    cases = next(m.args[1] for m in sort.test_sort.pytestmark if m.name == "parametrize" and m.args[0] == "T,k,E")
    assert set(kernels_of([("sort", T, k, E) for T, k, E in cases])) == {"sort one chunk 1"} | {f"sort chunks {r}" for r in (1, 2, 4, 8)}
