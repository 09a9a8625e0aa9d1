"""The host code of a mixture-of-experts layer's training operators under AddressSanitizer and UndefinedBehaviorSanitizer, without a GPU: a build of their
sources (and of the one that holds contexts and errors) with the sanitizers on the host pass only, walked by
tests/host_sanitize_moe_train.c.  Kept under _build/ and reused while the sources are unchanged."""
import hashlib
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_20313_amd", "csrc")
HIPCC = "/opt/rocm/bin/hipcc"
CLANG = "/opt/rocm/llvm/bin/clang"
DRIVER = os.path.join(ROOT, "tests", "host_sanitize_moe_train.c")


def digest():
    h = hashlib.sha256()
    for f in sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC)) + [os.path.join(ROOT, "include", "tilelink_mi355.h"), DRIVER]:
        h.update(open(f, "rb").read())
    return h.hexdigest()[:16]


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="needs the ROCm compilers")
def test_moe_train_host_code_is_clean_under_asan_and_ubsan():
    out = os.path.join(ROOT, "_build", "asan_moe_train")
    tag, lib, drv = (os.path.join(out, x) for x in ("digest", "libtilelink_moe_train_asan.so", "host_sanitize_moe_train"))
    if not (os.path.exists(tag) and open(tag).read() == digest() and os.path.exists(lib) and os.path.exists(drv)):
        shutil.rmtree(out, ignore_errors=True)
        os.makedirs(out)
        san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]

        def compile_one(name):
            obj = os.path.join(out, name + ".o")
            subprocess.run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"] + san +
                           ["-c", os.path.join(CSRC, name), "-o", obj], check=True, capture_output=True, timeout=900)
            return obj

        with ThreadPoolExecutor(3) as ex:
            objs = list(ex.map(compile_one, ["tl_dense.hip", "tl_moe_rows.hip", "tl_moe_products.hip"]))
        subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC"] + san + ["-o", lib] + objs, check=True, capture_output=True, timeout=300)
        subprocess.run([CLANG, "-fsanitize=address,undefined", "-g", "-I", os.path.join(ROOT, "include"), DRIVER, "-o", drv, "-L", out, "-ltilelink_moe_train_asan",
                        f"-Wl,-rpath,{out}", "-Wl,-rpath,/opt/rocm/lib"], check=True, capture_output=True, timeout=300)
        open(tag, "w").write(digest())
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([drv], capture_output=True, text=True, timeout=600, env=env)
    text = r.stdout + r.stderr
    assert r.returncode == 0, text[-3000:]
    assert "host_sanitize_moe_train ok" in r.stdout
    assert "AddressSanitizer" not in text and "runtime error" not in text and "LeakSanitizer" not in text, text[-3000:]
