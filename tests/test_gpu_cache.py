"""Block tables and slots (whole numbers: equal to the definition) and new keys and values in the paged
8-bit cache (every step is exact or a defined rounding: equal to the definition, byte for byte)."""
import dataclasses

import numpy as np
import pytest

from paper_2505_22654_amd import binding as vb
from paper_2505_22654_amd import workloads as wl
from tests import decode_reference as ref

pytestmark = pytest.mark.gpu


def _i32(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _plan_case(B, n_new, block, max_blocks, seed, spare=5, head=2):
    rng = np.random.default_rng(seed)
    cap = block * max_blocks
    new = rng.integers(0, n_new + 1, B) if n_new else np.zeros(B, int)
    cached = np.array([rng.integers(0, cap - n + 1) for n in np.minimum(new, cap)])
    if B:
        new[0] = n_new
        cached[0] = 0
    shape = wl.CacheShape("bf16", B, 1, 1, 64, block, 1, max_blocks, n_new)
    need = sum(-(-(c + min(n, cap - c)) // block) - -(-c // block) for c, n in zip(cached, new))
    used = sum(-(-c // block) for c in cached)
    total = used + need + spare + head
    order = rng.permutation(total)
    table = np.full((B, max_blocks), -7)
    at = 0
    for b, c in enumerate(cached):
        k = -(-c // block)
        table[b, :k] = order[at:at + k]
        at += k
    return dataclasses.replace(shape, n_blocks=int(total)), cached.tolist(), new.tolist(), order[at:].tolist(), head, table.tolist()


def _check_plan(shape, cached, new, free, head, table, **kw):
    import torch
    got = vb.cache_plan(shape, _i32(cached), _i32(new), _i32(free), _i32([head]), _i32(table).view(shape.batch, -1), **kw)
    want = ref.plan(shape, cached, new, free, head, table)
    torch.cuda.synchronize()
    assert got["block_table"].tolist() == want[0]
    assert got["slot_map"].tolist() == want[1]
    assert got["kv_len"].tolist() == want[2]
    assert (int(got["free_head"]), int(got["missing"])) == want[3:]
    return got


@pytest.mark.parametrize("B,n_new,block,max_blocks", [
    (1, 1, 16, 1), (1, 16, 16, 1), (3, 17, 16, 4), (5, 1, 256, 3), (64, 7, 32, 20), (256, 1, 16, 40),
    (1024, 4, 16, 9), (1025, 1, 64, 5), (2500, 1, 16, 3), (3000, 2, 16, 3), (33, 700, 128, 8), (2, 5000, 16, 400),
    (7, 1025, 16, 70), (1, 0, 16, 2),
])
def test_plan_matches_the_definition(B, n_new, block, max_blocks):
    _check_plan(*_plan_case(B, n_new, block, max_blocks, seed=B * 31 + n_new))


@pytest.mark.parametrize("B,n_new", [(5, 3), (40, 300)])
def test_plan_without_enough_blocks_hands_out_nothing(B, n_new):
    case = _plan_case(B, n_new, 16, 30, seed=8, spare=0)
    _check_plan(*case)                                           # the last block is handed out
    shape, cached, new, free, head, table = case
    got = _check_plan(shape, cached, new, free[:-1], head, table)
    assert int(got["missing"]) == 1 and int(got["free_head"]) == head
    got = _check_plan(shape, cached, new, [], 0, table)
    assert int(got["missing"]) >= 1


@pytest.mark.parametrize("B,n_new", [(1024, 1), (1024, 5), (1025, 5), (300, 40), (4, 9000), (2000, 2), (1, 300000)])
@pytest.mark.parametrize("missing", [0, 1])
def test_plan_in_place_and_beside(B, n_new, missing):
    """The lengths and the head overwritten, one of them, and neither: one result."""
    shape, cached, new, free, head, table = _plan_case(B, n_new, 16, -(-n_new // 16) + 3, seed=B + n_new, spare=0)
    free = free[:len(free) - missing]
    for over in ((), ("kv_len",), ("free_head",), ("kv_len", "free_head")):
        c, h, t = _i32(cached), _i32([head]), _i32(table).view(B, -1)
        got = vb.cache_plan(shape, c, _i32(new), _i32(free), h, t, out={n: {"kv_len": c, "free_head": h}[n] for n in over})
        want = ref.plan(shape, cached, new, free, head, table)
        assert got["kv_len"].tolist() == want[2] and (int(got["free_head"]), int(got["missing"])) == want[3:]
        assert got["slot_map"].tolist() == want[1] and t.tolist() == want[0]
        assert c.tolist() == (want[2] if "kv_len" in over else cached)
        assert int(h) == (want[3] if "free_head" in over else head)


def test_plan_holds_lengths_and_blocks_inside_their_ranges():
    shape = wl.CacheShape("bf16", 6, 1, 1, 64, 16, 40, 4, 20)
    table = [[i * 4 + j for j in range(4)] for i in range(6)]
    table[5][0] = 40                                             # a block the cache does not have
    free = [39, 38, 37, 36, -1, 99, 35, 34, 33, 32]
    _check_plan(shape, [-5, 70, 64, 60, 2 ** 31 - 1, 3], [25, 3, 1, 20, 2 ** 31 - 1, -2 ** 31], free, 0, table)
    _check_plan(shape, [3, 0, 0, 0, 0, 3], [9, 0, 20, 17, 20, 9], free, -3, table)
    _check_plan(shape, [0] * 6, [0] * 6, free, 1 << 30, table)
    empty = dataclasses.replace(shape, batch=0)
    got = vb.cache_plan(empty, _i32([]), _i32([]), _i32(free), _i32([4]), _i32([]).view(0, 4))
    assert int(got["free_head"]) == 4 and int(got["missing"]) == 0


@pytest.mark.parametrize("B,n_new", [(9, 1), (9, 600)])
def test_plan_in_place_step_after_step(B, n_new):
    """cached_len = kv_len and one head, over several steps."""
    shape, cached, _, _, _, _ = _plan_case(B, n_new, 16, 200, seed=3)
    shape = dataclasses.replace(shape, n_blocks=2000)
    free = np.random.default_rng(1).permutation(2000).tolist()
    kv, head, table = _i32([0] * B), _i32([0]), _i32([[-1] * 200] * B)
    wkv, whead, wtable = [0] * B, 0, table.tolist()
    for step in range(4):
        new = [(b + step) % (n_new + 1) for b in range(B)]
        out = vb.cache_plan(shape, kv, _i32(new), _i32(free), head, table, out={"kv_len": kv, "free_head": head})
        wtable, slots, wkv, whead, missing = ref.plan(shape, wkv, new, free, whead, wtable)
        assert (out["slot_map"].tolist(), kv.tolist(), int(head), int(out["missing"])) == (slots, wkv, whead, missing)
        assert table.tolist() == wtable


# ------------------------------------------------------------------------------------ new tokens
def _fresh_cache(shape, seed):
    """A cache with values of earlier tokens, and garbage scales where a block is begun later."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = vb.cache_alloc(shape)
    for n in ("k", "v"):
        codes = torch.randint(0, 127, cache[n].shape, generator=g, device="cuda")
        sign = torch.randint(0, 2, cache[n].shape, generator=g, device="cuda") * 128
        cache[n].copy_(torch.where(codes == 0, 0, codes + sign).to(torch.uint8))
        cache[n + "_scale"].copy_(torch.exp2(torch.randint(-12, -5, cache[n + "_scale"].shape, generator=g, device="cuda").float()))
    return cache


def _slots(shape, cached, new, seed):
    """(slot_map as lists, table): blocks of every sequence in no order."""
    bs, rng = shape.block_size, np.random.default_rng(seed)
    order, at, out = rng.permutation(shape.n_blocks), 0, []
    for c, n in zip(cached, new):
        blocks = order[at:at + -(-(c + n) // bs)]
        at += len(blocks)
        out.append([int(blocks[(c + r) // bs]) * bs + (c + r) % bs if r < n else -1 for r in range(shape.n_new)])
    return out


def _check_store(shape, cache, k, v, slot_map):
    import torch
    before = {n: t.clone() for n, t in cache.items()}
    vb.cache_store(shape, k, v, slot_map, cache)
    torch.cuda.synchronize()
    for n, x in (("k", k), ("v", v)):
        values, scales = ref.read(before, shape, n).cpu(), before[n + "_scale"].double().cpu()
        ref.store(shape, x.cpu(), slot_map.cpu(), values, scales)
        assert torch.equal(cache[n + "_scale"].double().cpu(), scales), (shape, n)
        got = ref.read(cache, shape, n).cpu()
        assert torch.equal(got, values), (shape, n, int((got != values).sum()))


STORES = [
    # dtype, kv heads, dh, block, new rows, lengths before
    ("bf16", 4, 128, 16, 1, [0, 1, 3, 15, 16, 17, 40]),
    ("bf16", 2, 128, 16, 40, [0, 1, 3, 15, 16, 17]),
    ("f32", 3, 80, 32, 70, [0, 5, 31, 32, 33]),
    ("f32", 1, 8, 64, 3, [0, 61, 62, 63, 64]),
    ("bf16", 1, 72, 128, 300, [0, 1, 127, 130]),
    ("bf16", 2, 256, 256, 257, [0, 255]),
    ("f32", 2, 200, 16, 33, [7, 0]),
    ("bf16", 5, 64, 16, 16, [0, 8, 15]),
    ("bf16", 32, 40, 64, 1, [63, 64, 2]),
]


@pytest.mark.parametrize("dtype,heads,dh,block,n_new,cached", STORES, ids=lambda v: str(v).replace(" ", ""))
@pytest.mark.parametrize("gain", [0.02, 1.0, 300.0])
def test_store_matches_the_definition(dtype, heads, dh, block, n_new, cached, gain):
    """Ragged rows; `gain` decides whether the scales of continued blocks grow."""
    import torch
    B = len(cached)
    new = [n_new if b == 0 else max(0, n_new - 5 * b) for b in range(B)] if n_new > 1 else [1] * B
    blocks = sum(-(-(c + n) // block) for c, n in zip(cached, new)) + 2
    shape = wl.CacheShape(dtype, B, heads, heads, dh, block, blocks, 1, n_new)
    cache = _fresh_cache(shape, B)
    g = torch.Generator(device="cuda").manual_seed(n_new)
    k, v = (torch.randn((B, heads, n_new, dh), generator=g, device="cuda").mul(gain).to(vb._torch_dtype(dtype)) for _ in "kv")
    _check_store(shape, cache, k, v, _i32(_slots(shape, cached, new, 2)))


def test_store_of_zeros_extremes_and_ties():
    import torch
    shape = wl.CacheShape("f32", 1, 1, 1, 64, 16, 3, 3, 16)
    cache = _fresh_cache(shape, 1)
    k = torch.zeros((1, 1, 16, 64), device="cuda")
    v = torch.full_like(k, 448.0)                               # the largest value of scale 1
    v[0, 0, :, ::2] = torch.tensor([17.0, 19.0, 21.0, 23.0, 0.001953125, 0.0009765625, 0.00146484375, 1e-30], device="cuda").repeat(4)
    slots = _i32([list(range(16, 32))])
    _check_store(shape, cache, k, v, slots)
    assert float(cache["k_scale"][1]) == 2.0 ** -120 and float(cache["v_scale"][1]) == 1.0
    for x in (torch.finfo(torch.float32).max, 449.0, 2.0 ** -110, 1e-45):
        _check_store(shape, cache, torch.full_like(k, x), torch.full_like(k, -x), slots)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block,n_new,cached", [(16, 1, 3), (16, 40, 5), (64, 100, 0), (256, 300, 9)])
def test_store_holds_infinities_and_nan_as_nan(dtype, block, n_new, cached):
    """They leave the scale and their neighbours alone."""
    import torch
    shape = wl.CacheShape(dtype, 1, 2, 2, 72, block, 30, 30, n_new)
    g = torch.Generator(device="cuda").manual_seed(block)
    k, v = (torch.randn((1, 2, n_new, 72), generator=g, device="cuda").to(vb._torch_dtype(dtype)) for _ in "kv")
    odd = torch.rand(k.shape, generator=g, device="cuda") < 0.02
    odd[0, 0, 0, 7] = odd[0, 1, -1, 71] = True
    odd[0, 1, 0, :] = True                                       # a row of nothing else
    bad = torch.tensor([float("inf"), -float("inf"), float("nan")], device="cuda").to(k.dtype)
    bad = bad[torch.arange(k.numel(), device="cuda").view(k.shape) % 3]
    slots = _i32(_slots(shape, [cached], [n_new], 3))
    plain, got = _fresh_cache(shape, 1), _fresh_cache(shape, 1)
    vb.cache_store(shape, torch.where(odd, 0, k), torch.where(odd, 0, v), slots, plain)
    vb.cache_store(shape, torch.where(odd, bad, k), torch.where(odd, bad, v), slots, got)
    for n in "kv":
        assert torch.equal(plain[n + "_scale"], got[n + "_scale"])
        a, b = ref.read(plain, shape, n), ref.read(got, shape, n)
        want = torch.zeros(a.shape, dtype=torch.bool, device="cuda")
        for r, s in enumerate(slots[0].tolist()):
            want[s // block, :, s % block, :72] = odd[0, :, r]
        assert torch.equal(b.isnan(), want) and torch.equal(a[~want], b[~want])


def test_store_leaves_out_rows_it_cannot_place():
    """-1, slots outside the cache, rows that do not continue their block; other blocks stay."""
    import torch
    shape = wl.CacheShape("bf16", 4, 2, 2, 64, 16, 6, 3, 20)
    cache = _fresh_cache(shape, 4)
    k, v = (torch.randn((4, 2, 20, 64), device="cuda").bfloat16() for _ in "kv")
    slots = [[-1] * 20,                                          # nothing
             list(range(10, 16)) + list(range(96, 110)),         # the second block does not exist
             [33, 34, 36, 37] + [-1] * 16,                       # two rows, then a gap
             list(range(64, 80)) + [80, 81, 82, -1]]
    before = {n: t.clone() for n, t in cache.items()}
    vb.cache_store(shape, k, v, _i32(slots), cache)
    for n, x in (("k", k), ("v", v)):
        values, scales = ref.read(before, shape, n).cpu(), before[n + "_scale"].double().cpu()
        valid = [slots[0], slots[1][:6] + [-1] * 14, slots[2][:2] + [-1] * 18, slots[3]]
        ref.store(shape, x.cpu(), torch.tensor(valid), values, scales)
        assert torch.equal(ref.read(cache, shape, n).cpu(), values)
        assert torch.equal(cache[n + "_scale"].double().cpu(), scales)


def test_store_takes_the_rows_of_longer_slabs():
    """What an in-place prune returns: the first rows of every slab."""
    import torch
    shape = wl.CacheShape("bf16", 2, 3, 3, 64, 16, 8, 4, 21)
    cache = _fresh_cache(shape, 6)
    long = [torch.randn((2, 3, 50, 64), device="cuda").bfloat16() for _ in "kv"]
    slots = _i32(_slots(shape, [0, 4], [21, 19], 1))
    _check_store(shape, cache, long[0][:, :, :21], long[1][:, :, :21], slots)
    with pytest.raises(ValueError):
        vb.cache_store(shape, long[0][:, :, :21], long[1][:, :, :21].contiguous(), slots, cache)
    with pytest.raises(ValueError):
        vb.cache_store(shape, long[0][:, :, ::2][:, :, :21], long[1][:, :, ::2][:, :, :21], slots, cache)


@pytest.mark.parametrize("block", [16, 64])
def test_store_token_by_token_is_the_store_of_all(block):
    """With scales that only grow by powers of two, values written one at a time are those written at
    once, but for what became subnormal on the way."""
    import torch
    n = 2 * block
    shape = wl.CacheShape("f32", 1, 2, 2, 64, block, 4, 4, n)
    one = dataclasses.replace(shape, n_new=1)
    x = torch.randn((1, 2, n, 64), device="cuda") * torch.linspace(0.1, 4, n, device="cuda")[:, None]
    slots = _i32(_slots(shape, [0], [n], 5))
    whole, steps = _fresh_cache(shape, 1), _fresh_cache(shape, 2)
    vb.cache_store(shape, x, x, slots, whole)
    for t in range(n):
        vb.cache_store(one, x[:, :, t:t + 1].contiguous(), x[:, :, t:t + 1].contiguous(), slots[:, t:t + 1].contiguous(), steps)
    used = sorted({int(s) // block for s in slots.flatten().tolist()})
    for kind in "kv":
        a, b = (ref.read(c, shape, kind)[used] for c in (whole, steps))
        assert torch.equal(whole[kind + "_scale"][used], steps[kind + "_scale"][used])
        normal = a.abs() >= 2.0 ** -6
        assert torch.equal(a[normal], b[normal]) and float((a - b).abs().max()) <= 2.0 ** -9


def test_store_of_slabs_more_than_32_bits_apart():
    import torch
    shape = wl.CacheShape("bf16", 1, 2, 2, 64, 16, 4, 4, 20)
    rows = 5 * (1 << 30) // 128                                  # a slab of 5 GB
    far = torch.empty(rows * 64 + 20 * 64, dtype=torch.bfloat16, device="cuda")
    x = far.as_strided((1, 2, 20, 64), (2 * rows * 64, rows * 64, 64, 1))
    x.copy_(torch.randn((1, 2, 20, 64), device="cuda"))
    slots = _i32(_slots(shape, [3], [20], 2))
    _check_store(shape, _fresh_cache(shape, 5), x, x, slots)
