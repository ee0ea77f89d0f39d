"""Sizes at the ends of what the vscan_cache_* calls take, host only: refused where no grid covers them, whatever
32 bits make of sums with them.  No GPU."""
import ctypes
import dataclasses
import os
import subprocess
import sys

import pytest

from paper_2505_22654_amd import binding as vb
from tests.test_abi_decode import CACHE, _plan, _store
from tests.test_sanitized_host import ROOT, SAN

TOP = 2 ** 31 - 1
ONE = dataclasses.replace(CACHE, batch=1, q_heads=1, kv_heads=1)


@pytest.mark.parametrize("block", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("less", [0, 1, 7, 9, 14, 15, 31, 63, 127, 253, 254, 255, 256, 400])
def test_store_refuses_the_longest_calls(block, less):
    desc = vb.cache_desc(dataclasses.replace(ONE, block_size=block, n_new=TOP - less))
    runs = (TOP - less + block - 2) // block + 1
    assert 2 * runs >= 1 << 24
    limit = (1 << 24) * (4 if block <= 32 else 1)
    assert _store(desc, k=None) == (vb.VSCAN_ERR_UNSUPPORTED if 2 * runs >= limit else vb.VSCAN_ERR_NULL)


def test_store_takes_what_the_limit_leaves():
    for block, n_new in ((16, (1 << 29) - 48), (256, TOP - 768)):
        runs = (n_new + block - 2) // block + 1
        assert 2 * runs < (1 << 24) * (4 if block <= 32 else 1)
        assert _store(vb.cache_desc(dataclasses.replace(ONE, block_size=block, n_new=n_new)), k=None) == vb.VSCAN_ERR_NULL


def test_plan_sizes_of_the_longest_calls():
    n = ctypes.c_size_t(0)
    for n_new in (1_800_000_000, TOP - 500, TOP):
        desc = vb.cache_desc(dataclasses.replace(ONE, n_new=n_new))
        assert vb.lib().vscan_cache_plan_workspace_size(ctypes.byref(desc), ctypes.byref(n)) == vb.VSCAN_OK and n.value >= 16
        assert _plan(desc, ws=None) == vb.VSCAN_ERR_WORKSPACE


CHECK = r"""
#include <stdio.h>
#include <stdlib.h>
#include "decode.hpp"
using namespace vscan;
static void need(bool ok, int n) { if (!ok) { printf("n_new %d\n", n); abort(); } }
int main() {
    const int sizes[] = {1, 1023, 1024, 1025, 1 << 30, 1800000000, 2147483647 - 1023, 2147483647 - 1022, 2147483647};
    for (int n : sizes) {
        // every row once, by steps that stay inside their type
        const int parts = plan_table_parts(n);
        need(parts >= 1 && (int64_t)parts * kTableThreads * 4 >= n && (int64_t)(parts - 1) * kTableThreads * 4 < n, n);
        const uint32_t step = (uint32_t)parts * kTableThreads;
        uint32_t r = step - 1, last = r;
        int turns = 0;
        for (; r < (uint32_t)n; r += step, ++turns) last = r;
        need(turns <= 4 && (int64_t)last + step >= n && (int64_t)turns * step >= n - (int64_t)step, n);
        for (int b = 16; b <= 256; b *= 2) {
            const int64_t runs = store_runs(n, b);
            need((runs - 1) * b >= n - 1 && (runs - 2) * b < n, n);
        }
    }
    puts("sizes-ok");
}
"""


def test_sizes_that_the_launches_use_stay_inside_their_types(tmp_path):
    src, exe = tmp_path / "sizes.cpp", str(tmp_path / "sizes")
    src.write_text(CHECK)
    subprocess.check_call(["g++", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__",
                           "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "paper_2505_22654_amd", "csrc"), str(src), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and "sizes-ok" in r.stdout, r.stdout + r.stderr


DRIVER = """
import ctypes, dataclasses, sys
from paper_2505_22654_amd import binding as vb, workloads as wl
L = ctypes.CDLL(sys.argv[1])
vp = ctypes.c_void_p
L.vscan_cache_plan.argtypes = [ctypes.POINTER(vb.CacheDesc), vp, vp, vp, ctypes.c_int32] + [vp] * 7 + [ctypes.c_size_t, vp]
L.vscan_cache_store.argtypes = [ctypes.POINTER(vb.CacheDesc)] + [vp] * 8
L.vscan_cache_attend.argtypes = [ctypes.POINTER(vb.CacheDesc)] + [vp] * 10 + [ctypes.c_size_t, vp]
L.vscan_test_decode_window.argtypes = [vp, ctypes.c_size_t]
FAKE, WSP, TOP, calls = 0x7F0000001000, 0x500000000000, 2 ** 31 - 1, 0
for block in (16, 64, 256):
    for n_new in (1 << 29, 1 << 30, 1800000000, TOP - 2 * block, TOP - block, TOP - 15, TOP):
        s = wl.CacheShape("bf16", 1, 1, 1, 64, block, TOP // block, TOP // block, n_new)
        d, n = ctypes.byref(vb.cache_desc(s)), ctypes.c_size_t(0)
        assert L.vscan_cache_plan_workspace_size(d, ctypes.byref(n)) == 0
        L.vscan_test_decode_window(WSP, n.value)
        assert L.vscan_cache_plan(d, *[FAKE] * 3, 5, *[FAKE] * 6, WSP, n.value, None) == 0
        runs = (n_new + block - 2) // block + 1
        fits = 2 * runs < (1 << 24) * (4 if block <= 32 else 1)
        assert L.vscan_cache_store(d, *[FAKE] * 7, None) == (0 if fits else vb.VSCAN_ERR_UNSUPPORTED)
        assert L.vscan_cache_attend(d, *[FAKE] * 9, WSP, 1 << 40, None) == vb.VSCAN_ERR_UNSUPPORTED
        calls += 1
print("sanitized-ok", calls)
"""


def test_the_host_layer_is_clean_at_the_largest_sizes(tmp_path):
    """The sanitizer build of tests/test_sanitized_decode.py, driven where 32 bits end."""
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
    driver = tmp_path / "driver.py"
    driver.write_text(DRIVER)
    r = subprocess.run([sys.executable, str(driver), lib], env=env, capture_output=True, text=True, timeout=600, cwd=ROOT)
    assert r.returncode == 0, f"exit {r.returncode}\n{r.stdout[-2000:]}\n{r.stderr[-4000:]}"
    assert "sanitized-ok 21" in r.stdout
