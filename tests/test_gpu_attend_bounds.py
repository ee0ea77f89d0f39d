"""vscan_cache_attend where its arithmetic could go wrong: sums that cancel, logits and queries at the ends
of fp32's range, queries with entries far apart, and every compiled form.  Definition and bounds as in
`decode_reference.attend`."""
import pytest

from paper_2505_22654_amd import binding as vb
from paper_2505_22654_amd import workloads as wl
from tests import decode_reference as ref
from tests.test_gpu_attend import HALF_STEP, i32, make

pytestmark = pytest.mark.gpu


def _stored(shape, k, v, lens):
    """A cache with the rows of k and v [B,Hkv,L,dh], its table, and the rows as the cache holds them."""
    import dataclasses

    import torch
    B, L = shape.batch, k.shape[2]
    cache = vb.cache_alloc(shape)
    for n in "kv":
        cache[n].zero_()
        cache[n + "_scale"].fill_(1.0)
    per = -(-L // shape.block_size)
    assert per <= shape.max_blocks and B * per <= shape.n_blocks
    table = torch.full((B, shape.max_blocks), -1, dtype=torch.int32, device="cuda")
    new = dataclasses.replace(shape, n_new=L, max_len=0)
    plan = vb.cache_plan(new, i32([0] * B), i32(lens), i32(list(range(shape.n_blocks))), i32([0]), table)
    vb.cache_store(new, k, v, plan["slot_map"], cache)
    rows = {n: (ref.read(cache, shape, n) * cache[n + "_scale"].double()[..., None, None])[..., :shape.head_dim]
            for n in "kv"}
    return cache, table, rows


def _two_planes_bound(shape, q, rows, cache, table, lens):
    """(result, bound) in 64 bits of a bf16 call: what fp32 calls are held to, for three
    planes of 8 bits 2^-26 of a weight, and for two planes of fp16 in their place half a step of the second,
    2^-22 of a weight, or below fp16's normal numbers 2^-25, of a largest weight of 2^4: 2^-29 of values of at
    most 448 scales a key."""
    import dataclasses
    f32 = dataclasses.replace(shape, dtype="f32")
    want, bound = ref.attend(f32, q, rows["k"], rows["v"], cache["v_scale"], table, lens, None)
    size, _ = ref.attend(f32, q, rows["k"], rows["v"].abs(), cache["v_scale"], table, lens, None)
    return want, bound + 2.0 ** -22 * size + max(lens) * 448 * 2.0 ** -29 * float(cache["v_scale"].max())


def _sums_that_cancel(B, hq, hkv, dh, T, length):
    """Tokens in pairs of opposite values and of nearly the same weight: what is left is far below the
    parts, and the weights' rounding would show (2^-11 of the parts against the bound's 2^-18)."""
    import torch
    shape = wl.CacheShape("bf16", B, hq, hkv, dh, 16, B * (-(-length // 16)) + 1, -(-length // 16), T)
    g = torch.Generator(device="cuda").manual_seed(length)
    k = torch.randn((B, hkv, length, dh), generator=g, device="cuda").bfloat16()
    v = torch.randn((B, hkv, length, dh), generator=g, device="cuda").bfloat16()
    pairs = length // 2
    v[:, :, 1:2 * pairs:2] = -v[:, :, 0:2 * pairs:2]
    v[:, :, 2 * pairs:] = 0
    lens = [length, length - 1 if length % 2 else length] * (B // 2)
    cache, table, rows = _stored(shape, k, v, lens)
    q = (torch.randn((B, hq, T, dh), generator=g, device="cuda") * 0.01).bfloat16()
    got = vb.cache_attend(shape, q, cache, table, i32(lens))["out"]
    want, bound = _two_planes_bound(shape, q, rows, cache, table, lens)
    over = (got.double() - want).abs() - bound - HALF_STEP["bf16"] * want.abs()
    assert float(over.max()) <= 0, (shape, float(over.max()))


@pytest.mark.parametrize("hq,hkv,dh,T,length", [(4, 4, 128, 1, 40), (28, 4, 128, 1, 333), (8, 2, 64, 3, 65), (2, 1, 192, 8, 20),
                                               (16, 1, 256, 1, 700), (6, 3, 80, 1, 5000)])
def test_sums_that_cancel_keep_their_bits_in_few_rows(hq, hkv, dh, T, length):
    _sums_that_cancel(2, hq, hkv, dh, T, length)


@pytest.mark.parametrize("B,hq,hkv,dh,T,length", [(2, 4, 4, 128, 17, 40), (2, 28, 4, 128, 5, 333), (2, 8, 2, 64, 9, 65), (2, 2, 1, 192, 40, 50),
                                                  (2, 4, 2, 256, 33, 700), (2, 6, 3, 80, 100, 5000), (64, 8, 4, 128, 50, 100), (64, 4, 4, 64, 64, 90)])
def test_sums_that_cancel_keep_their_bits_in_many_rows(B, hq, hkv, dh, T, length):
    _sums_that_cancel(B, hq, hkv, dh, T, length)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 3, 40])
@pytest.mark.parametrize("length", [1, 70, 3000])
def test_logits_far_below_zero(dtype, T, length):
    """Every logit between -1.4e36 and -2e31.  One token, which every row sees that sees any, has half the others':
    its value is the result."""
    import torch
    shape = wl.CacheShape(dtype, 2, 4, 2, 64, 16, 420, 200, T)
    g = torch.Generator(device="cuda").manual_seed(length)
    dt = vb._torch_dtype(dtype)
    k = torch.full((2, 2, length, 64), -64.0, device="cuda")
    first = max(length - T, 0)
    k[:, :, first] = -32.0
    v = torch.randn((2, 2, length, 64), generator=g, device="cuda").to(dt)
    lens = [length, length]
    cache, table, rows = _stored(shape, k.to(dt), v, lens)
    at = table.long()[:, first // 16]
    want = rows["v"][at, :, first % 16]                                    # [B, Hkv, dh]
    for gain in (2.0 ** 96, 2.0 ** 111):
        # 64 products of 32 gain or 64 gain, over 8: -256 gain and -512 gain
        q = torch.full((2, 4, T, 64), gain, device="cuda").to(dt)
        got = vb.cache_attend(shape, q, cache, table, i32(lens))["out"].double()
        seen = got[:, :, max(T - length, 0):]
        assert bool((seen == want.repeat_interleave(2, 1)[:, :, None].to(dt).double()).all()), (gain, seen)
        assert not got[:, :, :max(T - length, 0)].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 3, 40])
@pytest.mark.parametrize("length,present", [(1, True), (70, True), (3000, True), (70, False)])
def test_an_infinite_query_is_nan_also_where_every_logit_is_minus_infinity(dtype, T, length, present):
    """Keys of one sign in the dim where the query is infinite; rows without a key stay zero, the others as
    they are."""
    import torch
    shape = wl.CacheShape(dtype, 2, 4, 2, 64, 16, 420, 200, T)
    g = torch.Generator(device="cuda").manual_seed(length)
    k = torch.randn((2, 2, length, 64), generator=g, device="cuda")
    k[..., 5] = 0.5 + k[..., 5].abs()
    k, v = k.to(vb._torch_dtype(dtype)), torch.randn((2, 2, length, 64), generator=g, device="cuda").to(vb._torch_dtype(dtype))
    lens = [length, 0]
    cache, table, rows = _stored(shape, k, v, lens)
    if not present:
        table.fill_(-1)
    q = torch.randn((2, 4, T, 64), generator=g, device="cuda").to(vb._torch_dtype(dtype))
    want = vb.cache_attend(shape, q, cache, table, i32(lens))["out"]
    q[:, 1, T - 1, 5] = -float("inf")
    q[:, 2, 0, 5] = -float("inf")
    got = vb.cache_attend(shape, q, cache, table, i32(lens))["out"]
    odd = torch.zeros((2, 4, T), dtype=torch.bool, device="cuda")
    if present:
        odd[0, 1, T - 1] = True
        odd[0, 2, 0] = length >= T
    assert torch.equal(got[~odd], want[~odd]) and not want.isnan().any()
    assert bool(got[odd].isnan().all())
    assert not got[1].any() and (present or not got.any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,dh,T", [(4, 2, 64, 1), (8, 1, 256, 1), (4, 2, 128, 3), (4, 2, 128, 40), (2, 1, 192, 70)])
@pytest.mark.parametrize("length", [33, 1500])
def test_queries_at_the_top_of_the_range(dtype, hq, hkv, dh, T, length):
    """Queries of 2^119 to 2^126 and keys of 2^-114: products with the keys as they are stored, up to 448, pass
    fp32's range, the logits are of order 1 (the scale is 2^-9).  Other rows, and in fp32 entries of the largest
    fp32 number, which no bf16 number is near: the keys are 2^-129 there."""
    import torch
    shape = wl.CacheShape(dtype, 2, hq, hkv, dh, 16, 2 * (-(-length // 16)) + 1, -(-length // 16), T, scale=2.0 ** -9)
    g = torch.Generator(device="cuda").manual_seed(length + T)
    dt = vb._torch_dtype(dtype)
    k = torch.randn((2, hkv, length, dh), generator=g, device="cuda") * 2.0 ** -114
    q = torch.randn((2, hq, T, dh), generator=g, device="cuda") * 2.0 ** 124
    q = torch.where(q.abs() < 2.0 ** 119, 2.0 ** 119, q)
    if dtype == "f32":
        k[..., 7] = torch.where(k[..., 7] > 0, 2.0 ** -129, -(2.0 ** -129))
        q[..., 7] = torch.where(q[..., 7] > 0, 1.0, -1.0) * torch.finfo(torch.float32).max
    q[:, hq - 1] *= 2.0 ** -20                        # rows that would do without
    v = torch.randn((2, hkv, length, dh), generator=g, device="cuda").to(dt)
    lens = [length, 17]
    cache, table, rows = _stored(shape, k.to(dt), v, lens)
    q = q.to(dt)
    got = vb.cache_attend(shape, q, cache, table, i32(lens))["out"]
    want, bound = ref.attend(shape, q, rows["k"], rows["v"], cache["v_scale"], table, lens, None)
    assert bool(torch.isfinite(got).all())
    over = (got.double() - want).abs() - bound - HALF_STEP[dtype] * want.abs()
    assert float(over.max()) <= 0, float(over.max())
    # weights are spread, so that a wrong logit shows
    assert float((got.double() - want).norm() / want.norm()) < 0.02 and bool(want.any())


@pytest.mark.parametrize("B,hq,hkv,dh,T,length", [(2, 4, 2, 128, 40, 90), (2, 8, 1, 64, 30, 1500), (2, 2, 1, 256, 70, 300),
                                                  (2, 4, 2, 192, 33, 2600), (64, 8, 4, 128, 50, 100), (1, 2, 2, 72, 300, 2400)])
@pytest.mark.parametrize("apart", [8, 14, 20, 40, 126])
def test_queries_with_one_entry_far_above_the_others(B, hq, hkv, dh, T, length, apart):
    """An entry 2^apart of the others', in a dim where the keys are 0 or, in the last fifth of the tokens, whose
    keys are 2^8 times larger, as small as the format holds: the logits are those of the other entries."""
    import torch
    per = -(-length // 16)
    shape = wl.CacheShape("bf16", B, hq, hkv, dh, 16, B * per + 1, per, T)
    g = torch.Generator(device="cuda").manual_seed(apart + dh)
    k = torch.randn((B, hkv, length, dh), generator=g, device="cuda")
    k[..., 7] = 0
    last = length * 4 // 5 // 16 * 16
    k[:, :, last:] *= 2.0 ** 8
    v = torch.randn((B, hkv, length, dh), generator=g, device="cuda").bfloat16()
    lens = [length - 3 * (b % 5) for b in range(B)]
    cache, table, rows = _stored(shape, k.bfloat16(), v, lens)
    q = torch.randn((B, hq, T, dh), generator=g, device="cuda") * 2.0 ** -6
    q[..., 7] = 2.0 ** (apart - 6)
    q[0, 0, 0, 7] = 0
    q = q.bfloat16()
    got = vb.cache_attend(shape, q, cache, table, i32(lens))["out"]
    want, bound = _two_planes_bound(shape, q, rows, cache, table, lens)
    over = (got.double() - want).abs() - bound - HALF_STEP["bf16"] * want.abs()
    assert float(over.max()) <= 0, float(over.max())


@pytest.mark.parametrize("hq,hkv,dh,T,length", [(16, 4, 24, 40, 400), (2, 2, 16, 257, 300), (8, 1, 192, 9, 1500), (4, 1, 128, 16, 60),
                                                (6, 2, 80, 33, 700), (2, 1, 256, 64, 200), (4, 4, 64, 33, 2000)])
@pytest.mark.parametrize("gain", [16.0, 64.0])
def test_logits_with_a_large_product_keep_the_small_ones(hq, hkv, dh, T, length, gain):
    """One dim of the queries `gain` times the others, as models have them: logits of up to some hundred, whose
    differences are held to fp32 sums, (dh + 8) 2^-24 of the products' sizes, whatever the largest is."""
    import torch
    per = -(-length // 16)
    shape = wl.CacheShape("bf16", 2, hq, hkv, dh, 16, 2 * per + 1, per, T)
    g = torch.Generator(device="cuda").manual_seed(dh + T)
    k = torch.randn((2, hkv, length, dh), generator=g, device="cuda").bfloat16()
    v = torch.randn((2, hkv, length, dh), generator=g, device="cuda").bfloat16()
    lens = [length, length - 7]
    cache, table, rows = _stored(shape, k, v, lens)
    q = torch.randn((2, hq, T, dh), generator=g, device="cuda") * 2
    q[..., 3] *= gain
    q = q.bfloat16()
    got = vb.cache_attend(shape, q, cache, table, i32(lens))["out"]
    want, bound = _two_planes_bound(shape, q, rows, cache, table, lens)
    over = (got.double() - want).abs() - bound - HALF_STEP["bf16"] * want.abs()
    assert float(over.max()) <= 0, (float(over.max()), int((over > 0).sum()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 3, 40])
@pytest.mark.parametrize("size", [20, 28, 34, 60, 100])
def test_large_logits_pick_a_key(dtype, T, size):
    """Logits of 2^size and their half, where a step of fp32 is more than what an exponential holds from 2^31 on: the
    key of the larger one has all weight, or its copies share it evenly."""
    import torch
    length = 333
    shape = wl.CacheShape(dtype, 2, 4, 2, 64, 16, 44, 21, T, scale=1.0)
    g = torch.Generator(device="cuda").manual_seed(size + T)
    dt = vb._torch_dtype(dtype)
    k = torch.rand((2, 2, length, 64), generator=g, device="cuda") * 0.4 + 0.1
    q = torch.rand((2, 4, T, 64), generator=g, device="cuda") + 0.5
    best = [0, 17, length - T]
    k[:, :, best] = 1.3125                                               # one number, in e4m3 too
    v = torch.randn((2, 2, length, 64), generator=g, device="cuda").to(dt)
    lens = [length, length]
    cache, table, rows = _stored(shape, k.to(dt), v, lens)
    q = (q * 2.0 ** (size - 6)).to(dt)
    got = vb.cache_attend(shape, q, cache, table, i32(lens))["out"].double()
    picked = torch.stack([rows["v"][table.long()[:, j // 16], :, j % 16] for j in best]).double()
    want = picked.mean(0).repeat_interleave(2, 1)[:, :, None].expand(-1, -1, T, -1)
    bound = picked.abs().mean(0).repeat_interleave(2, 1)[:, :, None] * (2.0 ** -22 + 80 * 2.0 ** -24) + HALF_STEP[dtype] * want.abs()
    assert bool(torch.isfinite(got).all()) and float(((got - want).abs() - bound).max()) <= 0
