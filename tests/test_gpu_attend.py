"""vscan_cache_attend against softmax attention in 64 bits over the values the cache holds.  Tolerance:
`decode_reference.attend` derives it; half a step of the result's type is added for its rounding."""
import dataclasses

import numpy as np
import pytest

from paper_2505_22654_amd import binding as vb
from paper_2505_22654_amd import workloads as wl
from tests import decode_reference as ref

pytestmark = pytest.mark.gpu
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def make(shape, lens, seed, gain=1.0, spread=3):
    """q, a cache whose blocks hold N(0, 1) values of several scales, and a table.  Everything that no
    token fills holds NaN: blocks nobody has, rows behind the last token, and scales of unused blocks."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    bs, dh = shape.block_size, shape.head_dim
    dp = (dh + 63) // 64 * 64
    cache = vb.cache_alloc(shape)
    order = np.random.default_rng(seed).permutation(shape.n_blocks)
    table, at = np.full((shape.batch, shape.max_blocks), -1), 0
    tokens = torch.zeros(shape.n_blocks, dtype=torch.long)
    for b, n in enumerate(lens):
        k = -(-n // bs)
        table[b, :k] = order[at:at + k]
        for i in range(k):
            tokens[order[at + i]] = min(bs, n - i * bs)
        at += k
    tokens = tokens.cuda()
    rows = {}
    for n in ("k", "v"):
        e = torch.randint(-7 - spread, -6, (shape.n_blocks, shape.kv_heads), generator=g, device="cuda")
        scale = torch.exp2(e.double())
        x = torch.randn((shape.n_blocks, shape.kv_heads, bs, dp), generator=g, device="cuda").double() * 2.0 ** 7
        x[..., dh:] = 0
        values = ref.e4m3_round(x.clamp(-448, 448))
        values = torch.where(values == 0, 0.0, values)
        codes = ref.codes(values, shape, n)
        held = (torch.arange(bs, device="cuda")[None] < tokens[:, None]).double()
        mark = ref.codes(held[:, None, :, None].expand(-1, shape.kv_heads, -1, dp).contiguous(), shape, n)
        cache[n].copy_(torch.where(mark == 0, 0x7f, codes).view(cache[n].shape))
        cache[n + "_scale"].copy_(torch.where(tokens[:, None] > 0, scale, float("nan")).float())
        rows[n] = (values * scale[..., None, None])[..., :dh]
    q = (torch.randn((shape.batch, shape.q_heads, shape.n_new, dh), generator=g, device="cuda") * gain).to(vb._torch_dtype(shape.dtype))
    return q, cache, torch.tensor(table, dtype=torch.int32, device="cuda"), rows


def i32(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def check(shape, q, cache, table, rows, lens, new, **kw):
    import torch
    kv = i32(lens)
    got = vb.cache_attend(shape, q, cache, table, kv, None if new is None else i32(new), **kw)["out"]
    want, bound = ref.attend(shape, q, rows["k"], rows["v"], cache["v_scale"], table, lens, new)
    torch.cuda.synchronize()
    over = (got.double() - want).abs() - bound - HALF_STEP[shape.dtype] * want.abs()
    assert bool(torch.isfinite(got).all()) and float(over.max()) <= 0, (shape, float(over.max()))
    return got, want


def run(dtype, hq, hkv, dh, block, T, lens, new=None, seed=1, max_len=0, **kw):
    blocks = sum(-(-n // block) for n in lens) + 3
    shape = wl.CacheShape(dtype, len(lens), hq, hkv, dh, block, blocks, max(1, max(-(-n // block) for n in lens)), T, max_len)
    q, cache, table, rows = make(shape, lens, seed, **kw)
    return check(shape, q, cache, table, rows, lens, new)


LENS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 130, 255, 256, 257, 1000]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,dh,block", [(4, 4, 128, 16), (28, 4, 128, 16), (7, 1, 64, 32), (8, 2, 80, 64),
                                            (6, 3, 8, 16), (17, 1, 72, 128), (4, 2, 192, 16), (2, 1, 256, 256),
                                            (40, 1, 128, 16), (72, 1, 64, 16), (34, 2, 200, 32)])
def test_single_tokens(dtype, hq, hkv, dh, block):
    run(dtype, hq, hkv, dh, block, 1, LENS, seed=hq)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,dh,block,T", [(4, 4, 128, 16, 5), (14, 2, 128, 16, 9), (4, 1, 64, 16, 33),
                                              (2, 2, 96, 32, 130), (8, 1, 256, 16, 40), (3, 3, 24, 64, 300)])
def test_several_tokens_see_the_keys_up_to_their_own(dtype, hq, hkv, dh, block, T):
    """Lengths below T leave the first queries without a key."""
    run(dtype, hq, hkv, dh, block, T, [0, 1, T - 1, T, T + 1, 64, 333, 700], seed=T)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [4, 70])
def test_ragged_batches(dtype, T):
    """Padding rows are zero; new_len outside its range is held inside it."""
    lens = [500, 33, 64, 7, 0, 1000, 100]
    new = [T, 1, 0, T, T, T - 1, T + 9]
    got, _ = run(dtype, 12, 4, 128, 16, T, lens, new, seed=3)
    for b, n in enumerate(new):
        assert not got[b, :, min(n, T):].any()
    got, want = run(dtype, 4, 2, 64, 16, T, [90, 80], [-5, T], seed=4)
    assert not got[0].any()


@pytest.mark.parametrize("hq,hkv,T", [(28, 4, 1), (8, 1, 2), (4, 4, 3), (16, 1, 20)])
def test_long_caches_in_chunks(hq, hkv, T):
    for dtype in ("bf16", "f32"):
        run(dtype, hq, hkv, 128, 16, T, [9000, 4100], seed=5)
        run(dtype, hq, hkv, 64, 64, T, [20000], seed=6)


def test_large_logits_and_scales_far_apart():
    """Softmax that all but picks one key, references raised many times, scales 2^-37 .. 2^-7."""
    for dtype in ("bf16", "f32"):
        run(dtype, 8, 2, 128, 16, 3, [700, 65], gain=8.0, seed=7)
        run(dtype, 4, 4, 64, 16, 1, [700, 65], spread=30, seed=8)


@pytest.mark.parametrize("T,lens", [(33, [3005, 3025]), (1, [3005, 40]), (4, [300, 2000])])
def test_scales_on_either_side_of_what_goes_with_the_values(T, lens):
    """Scales 2^-27 .. 2^-7 in one sequence, and softmax near one key."""
    run("bf16", 132 if T > 4 else 8, 4, 48, 16, T, lens, seed=50279, gain=4, spread=20)


@pytest.mark.parametrize("apart", [12, 30, 90])
@pytest.mark.parametrize("T", [1, 40])
def test_all_weight_on_blocks_of_small_values(apart, T):
    """Values of a few blocks are 2^-apart of the others', and the queries look at those blocks alone."""
    import torch
    for dtype in ("bf16", "f32"):
        lens = [600, 333]
        shape = wl.CacheShape(dtype, 2, 4, 2, 128, 16, 62, 40, T)
        q, cache, table, rows = make(shape, lens, 21, spread=0)
        small = torch.zeros(shape.n_blocks, dtype=torch.bool, device="cuda")
        small[table[0, [3, 17]].long()] = True
        small[table[1, [0, 20]].long()] = True
        cache["v_scale"][small] *= 2.0 ** -apart
        rows["v"][small] *= 2.0 ** -apart
        # keys of the small blocks along one direction, the others against it
        one = torch.zeros(128, dtype=torch.float64, device="cuda")
        one[::2] = 448.0
        for sign, at in ((1, small), (-1, ~small)):
            held = ref.read(cache, shape, "k")[at]
            new = torch.where(held.isnan(), held, sign * one.expand_as(held))
            codes = ref.codes(torch.where(new.isnan(), 0.0, new), shape, "k")
            mark = ref.codes(new.isnan().double(), shape, "k")
            part = torch.where(mark == 0, codes, 0x7f).view(cache["k"][at].shape)
            cache["k"][at] = part
        rows["k"] = (ref.read(cache, shape, "k") * cache["k_scale"].double()[..., None, None])[..., :128]
        rows["k"] = torch.where(rows["k"].isnan(), 0.0, rows["k"])
        q = (0.5 + 0.1 * torch.rand_like(q.float())).to(q.dtype)
        got, want = check(shape, q, cache, table, rows, lens, None)
        # logits are at least 2 * 64 * 0.5 * 3.5 / sqrt(128) = 19.8 apart: the others weigh 600 e^-19.8 at most
        assert float(want[:, :, -1].abs().max()) < 100 * 2.0 ** -apart + 5 * 600 * 2.5e-9 and got[:, :, -1].any()


def test_max_len_bounds_the_keys():
    import torch
    for T in (1, 40):
        got, _ = run("bf16", 8, 2, 128, 16, T, [700, 300, 64, 301], max_len=301, seed=9)
        assert torch.isfinite(got).all()


def test_lengths_outside_the_table_are_held_inside_it():
    shape = wl.CacheShape("bf16", 3, 4, 2, 64, 16, 20, 5, 2)
    q, cache, table, rows = make(shape, [80, 33, 80], 3)
    got = vb.cache_attend(shape, q, cache, table, i32([2 ** 31 - 1, -7, 81]))["out"]
    want = vb.cache_attend(shape, q, cache, table, i32([80, 0, 80]))["out"]
    assert bool((got == want).all()) and not got[1].any()


@pytest.mark.parametrize("T", [1, 50])
def test_blocks_outside_the_cache_are_not_there(T):
    import torch
    shape = wl.CacheShape("bf16", 3, 8, 4, 128, 16, 60, 20, T)
    lens = [300, 320, 40]
    q, cache, table, rows = make(shape, lens, 11)
    table[0, 3], table[0, 18] = -1, 60
    table[1, ::2] = 2 ** 31 - 1
    table[2, :] = -2 ** 31
    got, _ = check(shape, q, cache, table, rows, lens, None)
    assert not got[2].any()


def test_queries_zeros_give_the_mean_of_the_values():
    import torch
    shape = wl.CacheShape("f32", 1, 2, 1, 64, 16, 40, 33, 1)
    q, cache, table, rows = make(shape, [517], 2)
    got = vb.cache_attend(shape, torch.zeros_like(q), cache, table, i32([517]))["out"]
    j = torch.arange(517, device="cuda")
    mean = rows["v"][table[0].long()[j // 16], 0, j % 16].mean(0)
    assert float((got.double() - mean).abs().max()) <= 1e-5 * float(rows["v"].abs().mean())


def test_given_buffers_and_scale():
    import torch
    shape = wl.CacheShape("bf16", 1, 4, 4, 64, 16, 400, 400, 2, scale=0.37)
    q, cache, table, rows = make(shape, [6000], 5)
    ws = torch.full((vb.cache_attend_workspace_size(vb.cache_desc(shape)),), 255, dtype=torch.uint8, device="cuda")
    out = {"out": torch.full_like(q, float("nan"))}
    got, _ = check(shape, q, cache, table, rows, [6000], None, workspace=ws, out=out)
    assert got is out["out"]
    with pytest.raises(vb.VscanError):
        vb.cache_attend(shape, q, cache, table, i32([6000]), workspace=ws[:-256])
    with pytest.raises(ValueError):
        vb.cache_attend(shape, q.float(), cache, table, i32([6000]))
    with pytest.raises(ValueError):
        vb.cache_attend(shape, q, cache, table[:, :-1], i32([6000]))
    with pytest.raises(ValueError):
        vb.cache_attend(shape, q, {**cache, "v": cache["k"]}, table, i32([6000]))


def test_results_do_not_depend_on_the_run():
    import torch
    shape = wl.CacheShape("bf16", 4, 28, 4, 128, 16, 800, 200, 1)
    q, cache, table, rows = make(shape, [3000, 100, 2222, 5], 12)
    kv = i32([3000, 100, 2222, 5])
    first = vb.cache_attend(shape, q, cache, table, kv)["out"]
    for _ in range(3):
        assert torch.equal(vb.cache_attend(shape, q, cache, table, kv)["out"], first)


def _poison(shape, cache, rows, table, name, b, j, head, dim):
    """Makes dim `dim` of token j of sequence b a NaN in the cache, and 0 in the rows of the definition."""
    bs, dp = shape.block_size, (shape.head_dim + 63) // 64 * 64
    block = int(table[b, j // bs])
    flat = cache[name].view(shape.n_blocks, shape.kv_heads, -1)
    flat[block, head, ref.offset(name, j % bs, dim, dp)] = 0xff if j % 2 else 0x7f
    rows[name][block, head, j % bs, dim] = 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,dh,block,T,lens", [
    (4, 4, 128, 16, 5, [40, 5, 3000]), (8, 2, 64, 32, 4, [64, 3]), (6, 2, 128, 16, 70, [70, 400, 33]),
    (2, 1, 192, 64, 40, [41, 300]), (4, 2, 256, 16, 9, [9, 129]), (14, 2, 80, 16, 300, [300, 1200]), (32, 8, 128, 16, 64, [500] * 40)])
def test_nan_reaches_the_rows_that_see_it(dtype, hq, hkv, dh, block, T, lens):
    """NaN in values and keys of the new tokens and before: rows that stand before them, and other heads and
    sequences, do not have any; dims whose values are whole neither, where the keys are."""
    import torch
    blocks = sum(-(-n // block) for n in lens) + 3
    shape = wl.CacheShape(dtype, len(lens), hq, hkv, dh, block, blocks, max(-(-n // block) for n in lens), T)
    q, cache, table, rows = make(shape, lens, 77)
    want_nan = torch.zeros(q.shape, dtype=torch.bool, device="cuda")
    G, rng = hq // hkv, np.random.default_rng(5)
    places = [(0, lens[0] - 1, 0, 0, "v"), (0, max(lens[0] - T, 0), hkv - 1, dh - 1, "v"), (1, lens[1] - 1, 0, dh // 2, "k")]
    for b, n in enumerate(lens):
        first = max(n - T, 0)
        places += [(b, int(rng.integers(first, n)), int(rng.integers(hkv)), int(rng.integers(dh)), "v") for _ in range(6)]
    if lens[-1] > 2 * T:
        places.append((len(lens) - 1, lens[-1] - T - 1, 0, 1, "v"))  # a token that every row sees
    for b, j, h, d, name in places:
        _poison(shape, cache, rows, table, name, b, j, h, d)
        t0 = max(j - (lens[b] - T), 0)
        want_nan[b, h * G:(h + 1) * G, t0:, slice(None) if name == "k" else d] = True
    got = vb.cache_attend(shape, q, cache, table, i32(lens))["out"]
    want, bound = ref.attend(shape, q, rows["k"], rows["v"], cache["v_scale"], table, lens, None)
    keyed = want_nan.all(-1, keepdim=True)
    assert torch.equal(got.isnan(), want_nan)
    over = (got.double() - want).abs() - bound - HALF_STEP[dtype] * want.abs()
    assert float(over[~want_nan & ~keyed].max()) <= 0


@pytest.mark.parametrize("T,lens", [(4, [30, 9, 2]), (70, [100, 70, 40]), (3, [5000, 4000, 1])])
def test_padding_rows_are_zero_whatever_they_hold(T, lens):
    import torch
    for dtype in ("bf16", "f32"):
        shape = wl.CacheShape(dtype, 3, 8, 2, 64, 16, sum(-(-n // 16) for n in lens) + 2, -(-max(lens) // 16), T)
        q, cache, table, rows = make(shape, lens, 12)
        new = [T - 1, 1, 0]
        for b, n in enumerate(new):
            q[b, :, n:] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device="cuda").to(q.dtype).repeat(16)
        got, _ = check(shape, torch.where(torch.isfinite(q) & (q.abs() < 1e38), q, 0), cache, table, rows, lens, new)
        again = vb.cache_attend(shape, q, cache, table, i32(lens), i32(new))["out"]
        assert torch.equal(got, again)
        for b, n in enumerate(new):
            assert not again[b, :, n:].any()


def test_two_calls_at_once_and_two_graphs():
    """Calls on two streams, eager and captured, each with its own workspace, and one workspace for calls
    that follow each other."""
    import torch
    shapes, states, want = [], [], []
    for i, (hq, hkv, dh, T, lens) in enumerate([(28, 4, 128, 1, [3000, 7, 2100]), (8, 2, 64, 50, [900, 60, 333])]):
        shapes.append(wl.CacheShape("bf16", 3, hq, hkv, dh, 16, sum(-(-n // 16) for n in lens) + 3, -(-max(lens) // 16), T))
        q, cache, table, rows = make(shapes[i], lens, 40 + i)
        states.append((q, cache, table, i32(lens)))
        want.append(check(shapes[i], q, cache, table, rows, lens, None)[0])
    streams = [torch.cuda.Stream() for _ in shapes]
    graphs, outs = [], []
    torch.cuda.synchronize()
    for sh, st, stream in zip(shapes, states, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            outs.append(vb.cache_attend(sh, *st)["out"])
        graphs.append(g)
    for _ in range(5):
        eager = []
        for i, stream in enumerate(streams):
            outs[i].fill_(-1)
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                graphs[i].replay()
                eager.append(vb.cache_attend(shapes[1 - i], *states[1 - i])["out"])
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i], want[i]) and torch.equal(eager[i], want[1 - i])
    need = max(vb.cache_attend_workspace_size(vb.cache_desc(sh)) for sh in shapes)
    space = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    for i in (0, 1, 0):
        got = vb.cache_attend(shapes[i], *states[i], workspace=space)["out"]
        assert torch.equal(got, want[i])


@pytest.mark.parametrize("T", [1, 40])
def test_sequences_that_share_blocks(T):
    """One prefix in the tables of several sequences, and a block twice in one table."""
    shape = wl.CacheShape("bf16", 3, 8, 2, 64, 16, 30, 12, T)
    q, cache, table, rows = make(shape, [150, 0, 0], 9)
    table[1:] = table[0]
    table[2, 5] = table[2, 1]
    check(shape, q, cache, table, rows, [150, 144, 97], None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_heads_of_one(dtype):
    run(dtype, 1024, 1, 64, 16, 1, [0, 40, 700])
    run(dtype, 300, 2, 72, 32, 3, [3, 1, 333])


def test_a_cache_of_more_than_32_bits():
    """The same tokens in blocks at either end of 5 GB: equal bit for bit."""
    import torch
    small = wl.CacheShape("bf16", 2, 8, 4, 128, 16, 40, 12, 150)
    large = dataclasses.replace(small, n_blocks=5 * (1 << 30) // (16 * 4 * 128))
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn((2, 4, 150, 128), generator=g, device="cuda").bfloat16() for _ in "kv")
    q = torch.randn((2, 8, 150, 128), generator=g, device="cuda").bfloat16()
    order = np.random.default_rng(4).permutation(small.n_blocks)
    far = [int(x) if x % 3 == 0 else large.n_blocks - 1 - int(x) for x in order]
    outs = []
    for shape, free in ((small, order.tolist()), (large, far)):
        cache = vb.cache_alloc(shape)
        table = torch.full((2, 12), -1, dtype=torch.int32, device="cuda")
        plan = vb.cache_plan(shape, i32([0, 0]), i32([150, 77]), i32(free), i32([0]), table)
        assert table.tolist()[0][:10] == free[:10]
        vb.cache_store(shape, k, v, plan["slot_map"], cache)
        one = dataclasses.replace(shape, n_new=1)
        outs.append([vb.cache_attend(shape, q, cache, table, plan["kv_len"], i32([150, 77]))["out"],
                     vb.cache_attend(one, q[:, :, :1].contiguous(), cache, table, plan["kv_len"])["out"]])
        for n in "kv":
            outs[-1].append(cache[n][table[table >= 0].long()].clone())
        del cache
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert bool(outs[0][0].any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 40])
def test_queries_of_wide_range(dtype, T):
    """Entries from 2^-30 to 2^5 in a row, rows from 2^-40 to 2^10, and a row of zeros."""
    import torch
    shape = wl.CacheShape(dtype, 2, 4, 2, 128, 16, 30, 14, T)
    q, cache, table, rows = make(shape, [200, 90], 21)
    g = torch.Generator(device="cuda").manual_seed(2)
    e = torch.randint(-30, 6, q.shape, generator=g, device="cuda").double()
    r = torch.randint(-40, 11, (2, 4, T, 1), generator=g, device="cuda").double()
    q = (q.double() * torch.exp2(e + r)).clamp(-3e4, 3e4).to(q.dtype)
    q[0, 0, 0] = 0
    check(shape, q, cache, table, rows, [200, 90], None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 40])
def test_a_query_that_is_not_finite_spoils_its_row_alone(dtype, T):
    import torch
    shape = wl.CacheShape(dtype, 2, 6, 2, 128, 16, 30, 14, T)
    q, cache, table, rows = make(shape, [200, 90], 5)
    want, _ = check(shape, q, cache, table, rows, [200, 90], None)
    odd = torch.zeros(q.shape[:3], dtype=torch.bool, device="cuda")
    odd[0, 1, T - 1] = odd[1, 5, 0] = odd[1, 2, 1] = True
    q[0, 1, T - 1, 3] = float("nan")
    q[1, 5, 0, 100] = float("inf")
    q[1, 2, 1, ::2] = -float("inf")
    got = vb.cache_attend(shape, q, cache, table, i32([200, 90]))["out"]
    assert torch.equal(got[~odd], want[~odd]) and bool(got[odd].isnan().all())
