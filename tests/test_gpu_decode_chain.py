"""The operators as they are used: rotate, prune, hand out blocks, store, then token after token."""
import dataclasses

import pytest

from paper_2505_22654_amd import binding as vb
from paper_2505_22654_amd import workloads as wl
from tests import decode_reference as ref
from tests.test_gpu_attend import HALF_STEP, i32

pytestmark = pytest.mark.gpu


class _Layer:
    """One layer's caches and request state for a batch."""

    def __init__(self, dtype, B, hq, hkv, dh, block, n_blocks, max_blocks, seed):
        import torch
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.dt, self.dh = vb._torch_dtype(dtype), dh
        self.shape = wl.CacheShape(dtype, B, hq, hkv, dh, block, n_blocks, max_blocks)
        self.cache = vb.cache_alloc(self.shape)
        self.table = torch.full((B, max_blocks), -1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(n_blocks, generator=self.g, device="cuda").int()
        self.head, self.kv = i32([0]), i32([0] * B)
        self.freq = vb.rope_frequencies(dh, 1e6)
        pairs = dh // 2
        self.sections = (pairs - 2 * (3 * pairs // 8), 3 * pairs // 8, 3 * pairs // 8)

    def rope(self, q, k, pos):
        B, S = self.shape.batch, k.shape[2]
        sh = wl.RopeShape(self.shape.dtype, B, S, q.shape[1], k.shape[1], self.dh, self.dh, self.sections)
        return vb.rope(sh, pos, self.freq, q, k), sh

    def rows(self):
        out = {}
        for n in ("k", "v"):
            out[n] = (ref.read(self.cache, self.shape, n) * self.cache[n + "_scale"].double()[..., None, None])[..., :self.dh]
        return out

    def attend(self, q, new_len=None):
        import torch
        sh = dataclasses.replace(self.shape, n_new=q.shape[2])
        got = vb.cache_attend(sh, q, self.cache, self.table, self.kv, new_len)["out"]
        rows = self.rows()
        want, bound = ref.attend(sh, q, rows["k"], rows["v"], self.cache["v_scale"], self.table, self.kv.tolist(), None if new_len is None else new_len.tolist())
        over = (got.double() - want).abs() - bound - HALF_STEP[sh.dtype] * want.abs()
        assert float(over.max()) <= 0, float(over.max())
        return got

    def randn(self, *size):
        import torch
        return torch.randn(size, generator=self.g, device="cuda").to(self.dt)


@pytest.mark.parametrize("dtype,in_place", [("bf16", 0), ("bf16", 1), ("f32", 0)])
def test_prompt_pruned_stored_and_continued(dtype, in_place):
    import torch
    B, hq, hkv, dh, block = 3, 8, 2, 64, 16
    prefix, vis, text, keep = 5, 48, 9, 17
    S = prefix + vis + text
    L = _Layer(dtype, B, hq, hkv, dh, block, 60, 8, 1)
    # positions on three axes: text, a 6 x 8 grid, text
    j = torch.arange(vis, device="cuda")
    text_pos = lambda a, n: torch.arange(a, a + n, device="cuda")[None].expand(3, n)  # noqa: E731
    pos = torch.cat([text_pos(0, prefix), prefix + torch.stack([j * 0, j // 8, j % 8]), text_pos(prefix + 8, text)], 1)
    pos = pos[:, None].expand(3, B, S).to(torch.int32).contiguous()
    q0, k0, v0 = L.randn(B, hq, S, dh), L.randn(B, hkv, S, dh), L.randn(B, hkv, S, dh)
    turned, rsh = L.rope(q0, k0, pos)
    llm = wl.LlmShape(dtype, B, prefix, vis, text, 1, hq, hkv, dh, 64, keep, in_place=in_place)
    k1, v1 = turned["k"].clone(), v0.clone()
    pruned = vb.llm_prune(llm, turned["q"][:, :, -1:].contiguous(), k1, v1, L.randn(B, S, 64))
    n = llm.seq_out
    sh = dataclasses.replace(L.shape, n_new=n)
    new = i32([n] * B)
    plan = vb.cache_plan(sh, L.kv, new, L.free, L.head, L.table, out={"kv_len": L.kv, "free_head": L.head})
    vb.cache_store(sh, pruned["k"], pruned["v"], plan["slot_map"], L.cache)
    assert int(plan["missing"]) == 0 and L.kv.tolist() == [n] * B
    # the cache holds the kept rows of the turned keys, rounded once
    kept = pruned["kept_idx"].long()
    rows = L.rows()
    for b in range(B):
        at = torch.cat([torch.arange(prefix, device="cuda"), prefix + kept[b], torch.arange(prefix + vis, S, device="cuda")])
        t = torch.arange(n, device="cuda")
        for name, x in (("k", ref.rope(k0, pos, L.freq, rsh)), ("v", v0.double())):
            got = rows[name][L.table[b].long()[t // block], :, t % block].transpose(0, 1)
            amax = x[b].abs().amax()
            # half a step of e4m3, half a step of the type and the rotation's own error; what is subnormal
            # under the scale (at most amax / 224 = 2 amax / 448) is off by half of 2^-9 of it
            tol = x[b, :, at].abs() * (2.0 ** -4 + 2.0 ** -7) + amax * (2.0 ** -10 * 2 / 448 + 2.0 ** -18)
            assert float(((got - x[b, :, at]).abs() - tol).max()) <= 0
    # tokens, one at a time; then a question of several tokens, ragged
    for step in range(20):
        one = L.shape
        p = i32([[[text + prefix + 8 + step]] * B] * 3)
        t, _ = L.rope(L.randn(B, hq, 1, dh), L.randn(B, hkv, 1, dh), p)
        plan = vb.cache_plan(one, L.kv, i32([1] * B), L.free, L.head, L.table, out={"kv_len": L.kv, "free_head": L.head})
        vb.cache_store(one, t["k"], L.randn(B, hkv, 1, dh), plan["slot_map"], L.cache)
        L.attend(t["q"])
    T, new = 11, i32([11, 3, 0])
    many = dataclasses.replace(L.shape, n_new=T)
    plan = vb.cache_plan(many, L.kv, new, L.free, L.head, L.table, out={"kv_len": L.kv, "free_head": L.head})
    vb.cache_store(many, L.randn(B, hkv, T, dh), L.randn(B, hkv, T, dh), plan["slot_map"], L.cache)
    out = L.attend(L.randn(B, hq, T, dh), new)
    assert not out[2].any() and not out[1, :, 3:].any()


def test_lengths_of_a_ragged_prune_feed_the_plan():
    import torch
    B, hq, hkv, dh = 3, 4, 4, 64
    caps = wl.LlmShape("bf16", B, 0, 60, 40, 1, hq, hkv, dh, 64, 20)
    meta = [(100, 10, 60, 20), (50, 3, 30, 7), (77, 0, 33, 0)]
    L = _Layer("bf16", B, hq, hkv, dh, 32, 30, 4, 2)
    S = caps.seq_len
    r = vb.llm_prune_ragged(caps, meta, L.randn(B, hq, 1, dh), L.randn(B, hkv, S, dh), L.randn(B, hkv, S, dh), L.randn(B, S, 64))
    sh = dataclasses.replace(L.shape, n_new=S)
    new = i32(r["out_len"])
    plan = vb.cache_plan(sh, L.kv, new, L.free, L.head, L.table, out={"kv_len": L.kv, "free_head": L.head})
    vb.cache_store(sh, r["k"], r["v"], plan["slot_map"], L.cache)
    assert L.kv.tolist() == r["out_len"]
    L.attend(L.randn(B, hq, 1, dh))
    L.attend(L.randn(B, hq, S, dh), new)


def test_steps_in_a_graph():
    """A decoding step captured once and replayed, with eager work between: each replay equals the
    eager step from the same state."""
    import torch
    B, hq, hkv, dh = 4, 28, 4, 128
    L = _Layer("bf16", B, hq, hkv, dh, 16, 900, 200, 3)
    start = [2100, 17, 0, 640]
    sh = dataclasses.replace(L.shape, n_new=max(start))
    plan = vb.cache_plan(sh, L.kv, i32(start), L.free, L.head, L.table, out={"kv_len": L.kv, "free_head": L.head})
    vb.cache_store(sh, L.randn(B, hkv, max(start), dh), L.randn(B, hkv, max(start), dh), plan["slot_map"], L.cache)
    one, rsh = L.shape, wl.RopeShape("bf16", B, 1, hq, hkv, dh, dh, L.sections)
    q, k, v, pos = L.randn(B, hq, 1, dh), L.randn(B, hkv, 1, dh), L.randn(B, hkv, 1, dh), i32([[[0]] * B] * 3)
    ones = i32([1] * B)

    def step(state):
        t = vb.rope(rsh, pos, L.freq, q, k)
        p = vb.cache_plan(one, state["kv"], ones, L.free, state["head"], state["table"],
                          out={"kv_len": state["kv"], "free_head": state["head"]})
        vb.cache_store(one, t["k"], v, p["slot_map"], state["cache"])
        return vb.cache_attend(one, t["q"], state["cache"], state["table"], state["kv"])["out"]

    def copy():
        return {"kv": L.kv.clone(), "head": L.head.clone(), "table": L.table.clone(), "cache": {n: t.clone() for n, t in L.cache.items()}}

    eager, caught = copy(), copy()
    warm = copy()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(warm)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(caught)
    for i in range(20):
        for t in (q, k, v):
            t.copy_(L.randn(*t.shape))
        pos.fill_(3000 + i)
        graph.replay()
        want = step(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        for n in ("kv", "head", "table"):
            assert torch.equal(caught[n], eager[n])
        for n in eager["cache"]:
            used = eager["table"][eager["table"] >= 0].long()
            assert torch.equal(caught["cache"][n][used], eager["cache"][n][used]), (i, n)
    assert eager["kv"].tolist() == [n + 20 for n in start]


def test_profile_and_log_names():
    vb.profile_enable(True)
    try:
        vb.profile_read()
        L = _Layer("bf16", 2, 4, 4, 64, 16, 700, 300, 5)
        t, _ = L.rope(L.randn(2, 4, 1, 64), L.randn(2, 4, 1, 64), i32([[[1]] * 2] * 3))
        p = vb.cache_plan(L.shape, L.kv, i32([1, 1]), L.free, L.head, L.table)
        vb.cache_store(L.shape, t["k"], t["k"], p["slot_map"], L.cache)
        vb.cache_attend(L.shape, t["q"], L.cache, L.table, p["kv_len"])
        names = vb.profile_read()
    finally:
        vb.profile_enable(False)
    assert {"rope", "cache_plan", "cache_store", "cache_attend"} <= set(names)
