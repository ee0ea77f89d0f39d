"""Every compiled form of the attention over the cache that shares keys between two row waves, and every one of
the store: which runs is decided by sizes (`attend_form`, `launch_store_lanes`)."""
import numpy as np
import pytest

from paper_2505_22654_amd import binding as vb
from paper_2505_22654_amd import workloads as wl
from tests import test_gpu_attend_bounds as bounds
from tests.test_gpu_attend import run
from tests.test_gpu_cache import _check_store, _fresh_cache, _i32, _slots

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,block", [(64, 16), (40, 64), (80, 32), (128, 16), (160, 16), (192, 128), (200, 32), (256, 16)])
def test_many_rows_of_many_sequences(dtype, dh, block):
    """64 sequences of 4 kv heads and 100 rows: 512 blocks of 64 rows, so two row waves share keys (fp32 heads above
    192 take 16 rows at a time).  Lengths of 0 to 300, new tokens of 0 to 50."""
    rng = np.random.default_rng(dh)
    lens = rng.integers(0, 300, 64).tolist()
    new = rng.integers(0, 51, 64).tolist()
    lens[:4], new[:4] = [0, 49, 50, 299], [50, 50, 50, 50]
    run(dtype, 8, 4, dh, block, 50, lens, new, seed=dh + block)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,lens", [(64, [3000] * 8 + [700] * 8), (33, [129, 2000] * 8)])
def test_many_rows_with_chunks_and_without(dtype, T, lens):
    run(dtype, 16, 16, 64, 16, T, lens, seed=T)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [24, 64, 104, 128, 136, 160, 192, 256])
@pytest.mark.parametrize("block", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("n_new", [1, 7, 30, 70, 300])
def test_store_of_every_page(dtype, dh, block, n_new):
    """From one quad of tokens to whole pages held at once, and pages that are read a second time."""
    import torch
    cached = [0, 5, block - 1]
    new = [n_new, max(1, n_new - 3), max(1, n_new // 2)]
    blocks = sum(-(-(c + n) // block) for c, n in zip(cached, new)) + 1
    shape = wl.CacheShape(dtype, 3, 1, 1, dh, block, blocks, 1, n_new)
    g = torch.Generator(device="cuda").manual_seed(n_new + dh)
    k, v = (torch.randn((3, 1, n_new, dh), generator=g, device="cuda").mul(gain).to(vb._torch_dtype(dtype)) for gain in (0.02, 30.0))
    _check_store(shape, _fresh_cache(shape, dh), k, v, _i32(_slots(shape, cached, new, 2)))


@pytest.mark.parametrize("dh", [64, 128, 192, 256])
def test_uneven_queries_of_many_sequences(dh):
    """One entry of the queries far above the others, and queries at the top of the range, with two row waves."""
    bounds.test_queries_with_one_entry_far_above_the_others(64, 8, 4, dh, 50, 130, 20)
    bounds.test_queries_with_one_entry_far_above_the_others(64, 8, 4, dh, 50, 130, 10)
    bounds.test_queries_at_the_top_of_the_range("bf16", 256, 128, dh, 50, 50)


def test_small_entries_that_count_late_in_a_sequence():
    """Keys 2^20 times larger from 2000 tokens on: entries of the queries 2^-18 of the largest, in whose dim the keys
    are 0, do nothing in the first blocks and decide in later ones, in another batch of block numbers."""
    import torch
    for hq, hkv, dh in ((2, 1, 128), (2, 1, 256)):
        T, length = 40, 2800
        shape = wl.CacheShape("bf16", 1, hq, hkv, dh, 16, 176, 175, T, scale=2.0 ** -12)
        g = torch.Generator(device="cuda").manual_seed(dh)
        k = torch.randn((1, hkv, length, dh), generator=g, device="cuda")
        k[..., 7] = 0
        k[:, :, 2000:] *= 2.0 ** 20
        v = torch.randn((1, hkv, length, dh), generator=g, device="cuda").bfloat16()
        cache, table, rows = bounds._stored(shape, k.bfloat16(), v, [length])
        q = torch.randn((1, hq, T, dh), generator=g, device="cuda") * 2.0 ** -11
        q[..., 7] = 2.0 ** 7
        q = q.bfloat16()
        got = vb.cache_attend(shape, q, cache, table, _i32([length]))["out"]
        want, bound = bounds._two_planes_bound(shape, q, rows, cache, table, [length])
        over = (got.double() - want).abs() - bound - 2.0 ** -8 * want.abs()
        assert float(over.max()) <= 0, (dh, float(over.max()))
