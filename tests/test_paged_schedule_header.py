"""The checks of a schedule against the dims of a call, on the CPU: tests/host_paged_schedule.hip, built with the host compiler pass
alone, without optimisation (every load of the source is made) and with AddressSanitizer, against the built library (which resolves the dims)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2503_20313_amd")
HIPCC = "/opt/rocm/bin/hipcc"


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs the ROCm compiler")
def test_a_schedule_is_told_from_those_of_other_dims(tmp_path):
    exe = str(tmp_path / "host_paged_schedule")
    subprocess.run([HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O0", "-g", "-std=c++17", "-Xarch_host", "-fsanitize=address", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(PKG, "csrc"), os.path.join(ROOT, "tests", "host_paged_schedule.hip"), "-o", exe, "-L", PKG, "-ltilelink_mi355", f"-Wl,-rpath,{PKG}"],
                   check=True, capture_output=True, timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1"))
    text = r.stdout + r.stderr
    assert r.returncode == 0 and "host_paged_schedule ok" in r.stdout and "AddressSanitizer" not in text, text[-3000:]
