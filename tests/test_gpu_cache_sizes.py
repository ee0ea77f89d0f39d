"""Cache calls near the ends of their ranges, and the compiled forms of the store that ordinary shapes do not
reach."""
import pytest

from paper_2505_22654_amd import binding as vb
from paper_2505_22654_amd import workloads as wl
from tests.test_gpu_attend import i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_new", [1_800_000_000, 2 ** 31 - 1])
def test_plan_of_the_longest_rows(n_new):
    """Lengths in place, so that a second launch writes the slots: more rows than a quarter added to them
    leaves inside 31 bits.  Slots of the few tokens that are there, -1 everywhere else, and nothing around."""
    import torch
    shape = wl.CacheShape("bf16", 1, 1, 1, 64, 16, 40, 40, n_new)
    guard = 1 << 20
    held = torch.full((n_new + 2 * guard,), -7, dtype=torch.int32, device="cuda")
    slots = held[guard:guard + n_new].view(1, n_new)
    kv, head, table = i32([5]), i32([0]), torch.full((1, 40), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 39
    out = vb.cache_plan(shape, kv, i32([30]), i32(list(range(40))), head, table,
                        out={"kv_len": kv, "free_head": head, "slot_map": slots})
    torch.cuda.synchronize()
    assert kv.tolist() == [35] and head.tolist() == [2] and out["missing"].tolist() == [0]
    assert table[0, :3].tolist() == [39, 0, 1] and not (table[0, 3:] + 1).any()
    want = [39 * 16 + 5 + r for r in range(11)] + list(range(19))
    assert slots[0, :30].tolist() == want
    assert bool((held[:guard] == -7).all()) and bool((held[-guard:] == -7).all())
    for at in range(30, n_new, 1 << 28):
        assert bool((slots[0, at:at + (1 << 28)] == -1).all())
    del held, slots, out
    torch.cuda.empty_cache()


def test_store_refuses_slabs_that_a_descriptor_does_not_hold():
    """2^32 + 50 rows of 8 dims between the heads: cut to 32 bits that would be 50."""
    import torch
    rows = (1 << 32) + 50
    if torch.cuda.mem_get_info()[0] < 2 * (rows * 16 + (1 << 30)):
        pytest.skip("not enough memory")
    far = torch.empty(rows * 8 + 64, dtype=torch.bfloat16, device="cuda")   # (never read)
    x = far.as_strided((1, 2, 3, 8), (2 * rows * 8, rows * 8, 8, 1))
    shape = wl.CacheShape("bf16", 1, 2, 2, 8, 16, 2, 2, 3)
    cache = vb.cache_alloc(shape)
    with pytest.raises(ValueError, match="rows"):
        vb.cache_store(shape, x, x, i32([[0, 1, 2]]), cache)
    del far, x
    torch.cuda.empty_cache()
