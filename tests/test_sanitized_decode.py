"""CPU build of the host layer behind vscan_rope and the vscan_cache_* calls (kernel launchers replaced
by tests/decode_stubs.cpp) under AddressSanitizer and UndefinedBehaviorSanitizer.  No GPU."""
import os
import subprocess
import sys

from tests.test_sanitized_host import ROOT, SAN


def test_decode_host_layer_is_clean_under_asan_and_ubsan(tmp_path):
    lib, csrc = str(tmp_path / "libvscan_decode_san.so"), os.path.join(ROOT, "paper_2505_22654_amd", "csrc")
    here = os.path.join(ROOT, "tests")
    subprocess.check_call(["g++", *SAN, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                           "-Wno-unused-result", "-Wno-deprecated-declarations",
                           *[os.path.join(csrc, f) for f in ("api.cpp", "budget.cpp", "decode_api.cpp")],
                           *[os.path.join(here, f) for f in ("host_stubs.cpp", "decode_stubs.cpp")], "-o", lib,
                           "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"])
    asan = subprocess.check_output(["gcc", "-print-file-name=libasan.so"], text=True).strip()
    env = dict(os.environ, LD_PRELOAD=asan, PYTHONPATH=ROOT,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=0:exitcode=23",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1:exitcode=24")
    r = subprocess.run([sys.executable, os.path.join(here, "sanitized_decode_driver.py"), lib], env=env,
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, f"exit {r.returncode}\n{r.stdout[-2000:]}\n{r.stderr[-4000:]}"
    assert "sanitized-ok" in r.stdout and int(r.stdout.split()[-1]) > 200
