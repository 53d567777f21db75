"""The host code of the norm and rotation and of the paged 8-bit cache under the address and undefined-behaviour sanitizers: the
library's host side alone, built for the test's temporary folder, driven by tests/c/paged_checks.c through rejections and
launch shapes of all sizes.  On the CPU; nothing is launched."""
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NM = shutil.which("nm") or "/opt/rocm/llvm/bin/llvm-nm"
SAN = ["-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=undefined"]


def test_paged_checks_under_address_and_undefined_sanitizers(tmp_path):
    hipcc, clang = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "/opt/rocm/llvm/bin/clang"
    if not all(os.path.exists(p) for p in (hipcc, clang, NM)):
        pytest.skip("no ROCm compiler here")
    from paper_2405_12591_amd import build as B
    inc = ["-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2405_12591_amd", "csrc")]
    host = [f for s in SAN for f in ("-Xarch_host", s)]

    def compile_one(src):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        r = subprocess.run([hipcc, "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIC", "-g", *host, *inc, "-c", src, "-o", obj],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        return obj

    with ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        objs = list(pool.map(compile_one, B.sources()))
    lib, exe = str(tmp_path / "libdecoquant_host.so"), str(tmp_path / "paged_checks")
    # the device code that the host side would register: none
    names = subprocess.run([NM, "-u", *objs], capture_output=True, text=True, check=True).stdout.split()
    blank = tmp_path / "blank.c"
    blank.write_text("".join("const char %s[4096] __attribute__((aligned(4096))) = {0};\n" % n for n in sorted({n for n in names if n.startswith("__hip_fatbin")})))
    objs.append(str(tmp_path / "blank.o"))
    subprocess.run([clang, "-fPIC", "-c", str(blank), "-o", objs[-1]], check=True)
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-fno-gpu-sanitize", *SAN, "-shared-libsan", *objs, "-o", lib],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([clang, "-std=c11", "-g", "-fno-gpu-sanitize", *SAN, "-shared-libsan", "-Wno-unused-command-line-argument",
                        os.path.join(ROOT, "tests", "c", "paged_checks.c"), "-I", os.path.join(ROOT, "include"),
                        lib, "-Wl,-rpath," + str(tmp_path), "-Wl,-rpath,/opt/rocm/lib", "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    rt = subprocess.run([clang, "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True, text=True).stdout.strip()
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1",
               LD_LIBRARY_PATH=os.path.dirname(rt) + ":/opt/rocm/lib:" + os.environ.get("LD_LIBRARY_PATH", ""))
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0 and "paged checks ok" in run.stdout, (run.stdout + run.stderr)[-4000:]
    assert "runtime error" not in run.stderr and "AddressSanitizer" not in run.stderr, run.stderr[-4000:]
