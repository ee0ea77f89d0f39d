"""Host-only checks of vscan_rope and the vscan_cache_* calls: every call here is refused before a
launch or has nothing to do, so the fake pointers are never dereferenced."""
import ctypes
import dataclasses

import pytest
import torch

from paper_2505_22654_amd import binding as vb
from paper_2505_22654_amd import workloads as wl

FAKE = 0x7F0000001000
OK, NULL, SHAPE, DTYPE, ALIGN = vb.VSCAN_OK, vb.VSCAN_ERR_NULL, vb.VSCAN_ERR_SHAPE, vb.VSCAN_ERR_DTYPE, vb.VSCAN_ERR_ALIGN
WS, VERSION, UNSUPPORTED = vb.VSCAN_ERR_WORKSPACE, vb.VSCAN_ERR_VERSION, vb.VSCAN_ERR_UNSUPPORTED

ROPE = wl.RopeShape(dtype="bf16", batch=2, seq_len=40, q_heads=28, kv_heads=4, head_dim=128, rot_dim=128,
                    sections=(16, 24, 24))
CACHE = wl.CacheShape(dtype="bf16", batch=3, q_heads=28, kv_heads=4, head_dim=128, block_size=16, n_blocks=100,
                      max_blocks=30, n_new=5)


def test_descriptor_layout_matches_header():
    assert ctypes.sizeof(vb.RopeDesc) == 16 * 4 + 6 * 8
    assert ctypes.sizeof(vb.CacheDesc) == 13 * 4


def _rope(desc, q=FAKE, k=FAKE, pos=FAKE, freq=FAKE, qo=FAKE, ko=FAKE):
    return vb.lib().vscan_rope(ctypes.byref(desc) if desc is not None else None, q, k, pos, freq, qo, ko, None)


@pytest.mark.parametrize("change,status", [
    (dict(batch=-1), SHAPE), (dict(seq_len=-1), SHAPE), (dict(q_heads=-1), SHAPE), (dict(kv_heads=1025), SHAPE),
    (dict(head_dim=124), SHAPE), (dict(head_dim=264), SHAPE), (dict(rot_dim=0, sections=(0,)), SHAPE),
    (dict(rot_dim=136, sections=(68,)), SHAPE), (dict(rot_dim=60, sections=(30,)), SHAPE),
    (dict(sections=(16, 24, 23)), SHAPE), (dict(sections=(-1, 65)), SHAPE), (dict(inverse=2), SHAPE),
    (dict(order=2), DTYPE), (dict(pairing=-1), DTYPE),
    (dict(batch=1 << 13, seq_len=1 << 12), UNSUPPORTED),
])
def test_rope_rejects_bad_descriptors(change, status):
    assert _rope(vb.rope_desc(dataclasses.replace(ROPE, **change))) == status


def test_rope_rejects_bad_pointers_and_strides():
    desc = vb.rope_desc(ROPE)
    assert _rope(None) == NULL
    bad = vb.rope_desc(ROPE)
    bad.struct_size -= 8
    assert _rope(bad) == VERSION
    bad = vb.rope_desc(ROPE)
    bad.dtype = 3
    assert _rope(bad) == DTYPE
    bad = vb.rope_desc(ROPE)
    bad.n_axes = 5
    assert _rope(bad) == SHAPE
    bad.n_axes = 0
    assert _rope(bad) == SHAPE
    for kw in (dict(q=None), dict(k=None), dict(pos=None), dict(freq=None)):
        assert _rope(desc, **kw) == NULL
    for kw in (dict(q=FAKE + 8), dict(k=FAKE + 2), dict(qo=FAKE + 4), dict(ko=FAKE + 8), dict(pos=FAKE + 2),
               dict(freq=FAKE + 4)):
        assert _rope(desc, **kw) == ALIGN
    # strides: negative, not a multiple of 16 bytes, beyond what offsets hold
    for stride in ((-8, 128, 128), (1 << 20, 128, 4), (1 << 35, 128, 1024)):
        assert _rope(vb.rope_desc(ROPE, q_stride=stride)) == SHAPE
        assert _rope(vb.rope_desc(ROPE, k_stride=stride)) == SHAPE
    # in place rows must not share memory; the same strides can be read from
    shared = vb.rope_desc(ROPE, k_stride=(4 * 40 * 128, 0, 128))
    assert _rope(shared, ko=None) == SHAPE
    assert _rope(shared, pos=None) == NULL       # past the stride check
    lapped = vb.rope_desc(ROPE, k_stride=(4 * 40 * 128, 40 * 128, 64))
    assert _rope(lapped, ko=None) == SHAPE
    woven = vb.rope_desc(ROPE, k_stride=(40 * 36 * 128, 128, 36 * 128))
    assert _rope(woven, ko=None, pos=None) == NULL


def test_rope_with_nothing_to_do():
    for change in (dict(batch=0), dict(seq_len=0), dict(q_heads=0, kv_heads=0)):
        assert _rope(vb.rope_desc(dataclasses.replace(ROPE, **change)), None, None, None, None, None, None) == OK


def _plan(desc, n_free=10, ws=FAKE, ws_bytes=1 << 30, **kw):
    a = dict(cached=FAKE, new=FAKE, free=FAKE, head=FAKE, table=FAKE, slots=FAKE, kv=FAKE, head_out=FAKE, missing=FAKE)
    a.update(kw)
    return vb.lib().vscan_cache_plan(ctypes.byref(desc) if desc is not None else None, a["cached"], a["new"], a["free"],
                                     n_free, a["head"], a["table"], a["slots"], a["kv"], a["head_out"], a["missing"],
                                     ws, ws_bytes, None)


def _store(desc, k=FAKE, v=FAKE, slots=FAKE, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE):
    return vb.lib().vscan_cache_store(ctypes.byref(desc) if desc is not None else None, k, v, slots, kc, vc, ks, vs, None)


def _attend(desc, q=FAKE, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, table=FAKE, kv=FAKE, new=FAKE, out=FAKE, ws=FAKE,
            ws_bytes=1 << 40):
    return vb.lib().vscan_cache_attend(ctypes.byref(desc) if desc is not None else None, q, kc, vc, ks, vs, table, kv,
                                       new, out, ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(batch=-1), SHAPE), (dict(batch=65536), SHAPE), (dict(n_blocks=0), SHAPE), (dict(max_blocks=0), SHAPE),
    (dict(n_new=-1), SHAPE), (dict(q_heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(q_heads=30), SHAPE),
    (dict(q_heads=1028), SHAPE), (dict(head_dim=100), SHAPE), (dict(head_dim=264), SHAPE),
    (dict(block_size=8), SHAPE), (dict(block_size=48), SHAPE), (dict(block_size=512), SHAPE),
    (dict(max_len=-1), SHAPE), (dict(max_len=481), SHAPE),
    (dict(n_blocks=1 << 27), SHAPE), (dict(max_blocks=1 << 27), SHAPE),
    (dict(batch=60000, max_blocks=1 << 16), UNSUPPORTED), (dict(batch=60000, n_new=1 << 16), UNSUPPORTED),
    (dict(n_blocks=(1 << 27) - 1, kv_heads=28), UNSUPPORTED),
])
def test_cache_calls_reject_bad_descriptors(change, status):
    desc = vb.cache_desc(dataclasses.replace(CACHE, **change))
    n, n2 = ctypes.c_size_t(0), ctypes.c_size_t(0)
    L = vb.lib()
    assert _plan(desc) == _store(desc) == _attend(desc) == status
    assert L.vscan_cache_size(ctypes.byref(desc), ctypes.byref(n), ctypes.byref(n2)) == status
    assert L.vscan_cache_plan_workspace_size(ctypes.byref(desc), ctypes.byref(n)) == status
    assert L.vscan_cache_attend_workspace_size(ctypes.byref(desc), ctypes.byref(n)) == status


def test_cache_calls_reject_bad_pointers_and_workspaces():
    desc = vb.cache_desc(CACHE)
    assert _plan(None) == _store(None) == _attend(None) == NULL
    for field, value, status in (("struct_size", 48, VERSION), ("dtype", 2, DTYPE), ("seq_len", 4, SHAPE), ("seq_len", -1, SHAPE)):
        bad = vb.cache_desc(CACHE)
        setattr(bad, field, value)
        assert _plan(bad) == _store(bad) == _attend(bad) == status
    for name in ("cached", "new", "free", "head", "table", "slots", "kv", "head_out", "missing"):
        assert _plan(desc, **{name: None}) == NULL
        assert _plan(desc, **{name: FAKE + 2}) == ALIGN
    assert _plan(desc, n_free=-1) == SHAPE
    # lengths of few rows stay in one workgroup, more need scratch
    assert vb.cache_plan_workspace_size(desc) == 0
    for change in (dict(batch=1025, n_new=0), dict(batch=8, n_new=513)):
        many = vb.cache_desc(dataclasses.replace(CACHE, **change))
        need = vb.cache_plan_workspace_size(many)
        assert need >= 16 * change["batch"]
        assert _plan(many, ws=None) == _plan(many, ws_bytes=need - 1) == WS
        assert _plan(many, ws=FAKE + 8) == ALIGN
    for name in ("k", "v", "slots", "kc", "vc", "ks", "vs"):
        assert _store(desc, **{name: None}) == NULL
        assert _store(desc, **{name: FAKE + 2}) == ALIGN
    for name in ("q", "kc", "vc", "ks", "vs", "table", "kv", "out"):
        assert _attend(desc, **{name: None}) == NULL
        assert _attend(desc, **{name: FAKE + 2}) == ALIGN
    assert _attend(desc, new=FAKE + 2) == ALIGN
    # many keys for few rows: cut into chunks, which need scratch
    long = vb.cache_desc(dataclasses.replace(CACHE, max_blocks=4096, batch=1))
    need = vb.cache_attend_workspace_size(long)
    assert need > 5 * 28 * 128 * 4
    assert _attend(long, ws=None) == _attend(long, ws_bytes=need - 1) == WS
    assert _attend(long, ws=FAKE + 8) == ALIGN
    for fn in ("vscan_cache_plan_workspace_size", "vscan_cache_attend_workspace_size"):
        assert getattr(vb.lib(), fn)(ctypes.byref(desc), None) == NULL


def test_cache_calls_refuse_grids_beyond_the_runtime():
    """2^32 threads: 2^24 workgroups of 256."""
    base = dataclasses.replace(CACHE, batch=1 << 12, q_heads=128, kv_heads=128, n_blocks=100, max_blocks=1 << 12)
    for block, n_new, ok in ((16, 16 * 61, True), (16, 16 * 64, False), (64, 64 * 13, True), (64, 64 * 16, False)):
        desc = vb.cache_desc(dataclasses.replace(base, block_size=block, n_new=n_new))
        assert _store(desc, slots=None) == (NULL if ok else UNSUPPORTED), (block, n_new)
    for n_new, ok in ((64 * 31, True), (64 * 32, False)):
        desc = vb.cache_desc(dataclasses.replace(base, n_new=n_new))
        assert _attend(desc, q=None) == (NULL if ok else UNSUPPORTED)


def test_cache_calls_with_nothing_to_do():
    none = vb.cache_desc(dataclasses.replace(CACHE, batch=0))
    assert _store(none, None, None, None, None, None, None, None) == OK
    assert _attend(none, None, None, None, None, None, None, None, None, None, None, 0) == OK
    empty = vb.cache_desc(dataclasses.replace(CACHE, n_new=0))
    assert _store(empty, None, None, None, None, None, None, None) == OK
    assert _attend(empty, None, None, None, None, None, None, None, None, None, None, 0) == OK


@pytest.mark.parametrize("dh,dp", [(8, 64), (64, 64), (72, 128), (128, 128), (136, 192), (200, 256), (256, 256)])
def test_cache_size(dh, dp):
    desc = vb.cache_desc(dataclasses.replace(CACHE, head_dim=dh))
    n, n2 = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert vb.lib().vscan_cache_size(ctypes.byref(desc), ctypes.byref(n), ctypes.byref(n2)) == OK
    assert (n.value, n2.value) == (100 * 4 * 16 * dp, 100 * 4 * 4)


def test_binding_refuses_tensors_it_cannot_use():
    pos = torch.zeros((3, 2, 40), dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        vb.rope(ROPE, pos, torch.zeros(64, dtype=torch.float64), torch.zeros(1), torch.zeros(1))
    with pytest.raises(ValueError, match="CUDA"):
        vb.cache_plan(CACHE, pos, pos, pos, pos, torch.zeros((3, 30), dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        vb.cache_store(CACHE, pos, pos, pos, {})
    with pytest.raises(ValueError, match="CUDA"):
        vb.cache_attend(CACHE, pos, {}, pos, pos)
    with pytest.raises(ValueError, match="axes"):
        vb.rope_desc(dataclasses.replace(ROPE, sections=(8, 8, 8, 8, 32)))
    with pytest.raises(vb.VscanError):
        vb.cache_alloc(dataclasses.replace(CACHE, block_size=17), "cpu")
