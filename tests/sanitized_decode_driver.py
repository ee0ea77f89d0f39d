"""Runs inside a child process whose runtime has AddressSanitizer preloaded (started by
tests/test_sanitized_decode.py, never collected by pytest).  argv: the sanitized CPU build of the host
layer.  Drives vscan_rope and the vscan_cache_* calls over drawn shapes with stand-in launchers that
check the scratch and grids handed to them.  Prints `sanitized-ok N` at the end."""
import ctypes
import random
import sys

from paper_2505_22654_amd import binding as vb
from paper_2505_22654_amd import workloads as wl

L = ctypes.CDLL(sys.argv[1])
vp, szp = ctypes.c_void_p, ctypes.POINTER(ctypes.c_size_t)
L.vscan_rope.argtypes = [ctypes.POINTER(vb.RopeDesc)] + [vp] * 7
L.vscan_cache_plan.argtypes = [ctypes.POINTER(vb.CacheDesc), vp, vp, vp, ctypes.c_int32] + [vp] * 7 + [ctypes.c_size_t, vp]
L.vscan_cache_store.argtypes = [ctypes.POINTER(vb.CacheDesc)] + [vp] * 8
L.vscan_cache_attend.argtypes = [ctypes.POINTER(vb.CacheDesc)] + [vp] * 10 + [ctypes.c_size_t, vp]
L.vscan_test_decode_window.argtypes = [vp, ctypes.c_size_t]
FAKE, WSP = 0x7F0000001000, 0x500000000000
rng, calls = random.Random(11), 0
for _ in range(400):
    kv = rng.choice((1, 2, 4, 8, 32))
    s = wl.CacheShape(rng.choice(("bf16", "f32")), rng.choice((0, 1, 3, 64, 2000)), kv * rng.choice((1, 2, 7, 8)), kv,
                      8 * rng.randint(1, 32), rng.choice((16, 32, 64, 128, 256)), rng.randint(1, 5000), rng.randint(1, 4000),
                      rng.choice((0, 1, 2, 7, 100, 2000)))
    d = ctypes.byref(vb.cache_desc(s))
    n = ctypes.c_size_t(0)
    assert L.vscan_cache_plan_workspace_size(d, ctypes.byref(n)) == 0
    L.vscan_test_decode_window(WSP, n.value)
    args = [d, FAKE, FAKE, FAKE, 5] + [FAKE] * 6 + [WSP]
    if n.value:
        assert L.vscan_cache_plan(*args, n.value - 1, None) == vb.VSCAN_ERR_WORKSPACE
    assert L.vscan_cache_plan(*args, n.value, None) == 0
    assert L.vscan_cache_store(d, *[FAKE] * 7, None) == 0
    rc = L.vscan_cache_attend_workspace_size(d, ctypes.byref(n))
    if rc == vb.VSCAN_ERR_UNSUPPORTED:
        assert s.batch * s.q_heads * s.n_new >= 1 << 21
        continue
    assert rc == 0
    L.vscan_test_decode_window(WSP, n.value)
    assert L.vscan_cache_attend(d, *[FAKE] * 9, WSP, n.value, None) == 0
    calls += L.vscan_test_decode_launches()
    rot = 8 * rng.randint(1, s.head_dim // 8)
    cut = rng.randint(0, rot // 2)
    r = wl.RopeShape(s.dtype, min(s.batch, 64), s.n_new, s.q_heads, kv, s.head_dim, rot, (cut, rot // 2 - cut, 0),
                     rng.randint(0, 1), rng.randint(0, 1), rng.randint(0, 1))
    out = [rng.choice((FAKE, None)) for _ in range(2)]
    assert L.vscan_rope(ctypes.byref(vb.rope_desc(r)), FAKE, FAKE, FAKE, FAKE, *out, None) == 0
print("sanitized-ok", calls)
