"""Performance cases: the steps around a pruned prefill as a serving program makes them.

Before `llm_prune` a layer's queries and keys are turned by their positions; after it the keys and
values that are left go into a paged cache of 8-bit values, and every later token is written to that
cache and attends over it.  A case is one call of one of these operators:

  op "rope"    rotary positions with one to three axes on q and k of a layer
  op "plan"    cache blocks handed to a batch of requests: block tables, slots, lengths
  op "store"   keys and values of new tokens into the cache, with a scale per block and kv head
  op "attend"  queries of the new tokens over the cache

`run` makes the framework's calls where `own` is true; otherwise it computes the same in elementary
torch operations.

The cache holds e4m3 values with a power-of-two scale per (block, kv head).  A block is made of groups
of 16 tokens; `dp` is head_dim rounded up to a multiple of 64 (the rest is zero):
  k  [n_blocks, kv_heads, block/16, dp/16, 16 tokens, 16 dims]
  v  [n_blocks, kv_heads, block/16, dp/64, 4, 16, 4, 4]: token 4*i4 + i7, dim 64*i3 + 16*i6 + i5
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_FP8 = torch.float8_e4m3fn
_MAX = 448.0            # largest e4m3 value
_EXP_LO, _EXP_HI = -120, 120
_DEV = "cuda"


# ------------------------------------------------------------------------------------- the cases
def _rope(name, dtype, batch, seq, q_heads, kv_heads, head_dim, sections, grid, qkv, inverse=False,
          cycled=False, adjacent=False, far=0):
    """`grid`: frames, rows and columns of the visual span ("t,h,w"); `qkv`: q and k are views of one
    projection output; `far`: position of the first token."""
    return {"name": name, "op": "rope", "dtype": dtype, "batch": batch, "seq": seq, "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "sections": sections, "grid": grid, "qkv": qkv,
            "inverse": inverse, "cycled": cycled, "adjacent": adjacent, "far": far}


def _plan(name, batch, new, cached, block):
    """Requests with up to `cached` tokens in the cache and up to `new` more."""
    return {"name": name, "op": "plan", "batch": batch, "new": new, "cached": cached, "block": block}


def _store(name, dtype, batch, new, cached, kv_heads, head_dim, block):
    return {"name": name, "op": "store", "dtype": dtype, "batch": batch, "new": new, "cached": cached,
            "kv_heads": kv_heads, "head_dim": head_dim, "block": block}


def _attend(name, dtype, batch, new, length, q_heads, kv_heads, head_dim, block):
    """Up to `length` tokens in the cache, the last `new` of them the queries'."""
    return {"name": name, "op": "attend", "dtype": dtype, "batch": batch, "new": new, "length": length,
            "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "block": block}


def listed():
    return [
        # one decoding step of 64 sequences, grouped heads, three axes: the smallest call
        _rope("rope-decode-64", "bf16", 64, 1, 28, 4, 128, "16,24,24", "1,1,1", True, far=4351),
        # a 64 x 64 visual grid and its text in one prompt, q and k as the projection leaves them
        _rope("rope-prompt-4352", "bf16", 1, 4352, 28, 4, 128, "16,24,24", "1,64,64", True),
        # gradient of an encoder's two-axis rotation, full precision, an odd grid
        _rope("rope-f32-inverse-2745", "f32", 2, 2745, 16, 16, 80, "20,20", "1,45,61", False, inverse=True),
        # one decoding step of 256 requests
        _plan("plan-decode-256", 256, 1, 3427, 16),
        # 32 prompts of up to 3427 tokens admitted at once
        _plan("plan-prompts-32", 32, 3427, 0, 16),
        # one decoding step's keys and values of a layer
        _store("store-decode-32", "bf16", 32, 1, 1267, 32, 128, 16),
        # what is left of 32 pruned prompts (35 + 720 + 512 tokens), the largest write
        _store("store-prompts-32", "bf16", 32, 1267, 0, 32, 128, 16),
        # one sequence, grouped heads, one token: latency counts
        _attend("attend-decode-1x2304", "bf16", 1, 1, 2304, 28, 4, 128, 16),
        # a decoding batch before the pruned layers, one kv head per query head: memory
        _attend("attend-decode-32x3427", "bf16", 32, 1, 3427, 32, 32, 128, 16),
        # few sequences with a long history
        _attend("attend-decode-4x65536", "bf16", 4, 1, 65536, 28, 4, 128, 64),
        # the next question of a dialogue: 300 new tokens over what is cached
        _attend("attend-turn-3x300", "bf16", 3, 300, 2604, 28, 4, 128, 16),
        # full precision, a head of 80, a few tokens at once
        _attend("attend-f32-5x4", "f32", 5, 4, 1391, 16, 8, 80, 32),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _sections(rng, pairs, axes):
    cuts = sorted(rng.sample(range(1, pairs), axes - 1)) if axes > 1 else []
    return ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [pairs]))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        dtype = rng.choice(("bf16", "bf16", "f32"))
        kv = rng.choice((1, 2, 3, 4, 8, 16, 32))
        group = rng.choice((1, 1, 2, 4, 7, 8)) if kv <= 8 else 1
        block = rng.choice((16, 16, 32, 64, 128, 256))
        op = rng.choice(("rope", "plan", "store", "store", "attend", "attend", "attend"))
        if op == "rope":
            dim = rng.choice((32, 64, 72, 80, 96, 128, 128, 256))
            axes = rng.choice((1, 2, 3))
            t, h, w = rng.randint(1, 4), rng.randint(1, 40), rng.randint(1, 40)
            text = _log_int(rng, 1, 2000)
            seq = rng.choice((1, t * h * w + text))
            case = _rope("", dtype, _log_int(rng, 1, 64), seq, kv * group, kv, dim,
                         _sections(rng, dim // 2, axes), "%d,%d,%d" % ((1, 1, 1) if seq == 1 else (t, h, w)),
                         rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.3, rng.random() < 0.3,
                         rng.choice((0, rng.randint(1, 200000))))
        elif op == "plan":
            new = rng.choice((1, _log_int(rng, 1, 4500)))
            case = _plan("", _log_int(rng, 1, 2000), new, rng.choice((0, _log_int(rng, 1, 20000))), block)
        elif op == "store":
            new = rng.choice((1, _log_int(rng, 1, 4500)))
            case = _store("", dtype, _log_int(rng, 1, 64), new, rng.choice((0, _log_int(rng, 1, 5000))), kv,
                          rng.choice((40, 64, 72, 80, 96, 128, 128, 256)), block)
        else:
            new = rng.choice((1, 1, _log_int(rng, 1, 1500)))
            case = _attend("", dtype, _log_int(rng, 1, 64), new, max(new, _log_int(rng, 1, 70000)), kv * group,
                           kv, rng.choice((40, 64, 72, 80, 96, 128, 128, 256)), block)
        del case["name"]
        if _cost(case) <= most and _size(case) <= 6e8:
            return case


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def _size(case):
    """Elements of the largest tensor of a plain pass: the logits of many queries, or the cache."""
    if case["op"] == "attend":
        return max(case["batch"] * case["q_heads"] * case["new"] * case["length"],
                   case["batch"] * case["kv_heads"] * case["length"] * case["head_dim"])
    if case["op"] == "store":
        return case["batch"] * case["kv_heads"] * (case["new"] + case["cached"]) * case["head_dim"]
    return 0


def _lengths(case):
    """Tokens (cached, new) of every request: the first has the most of both, the others are drawn."""
    rng = random.Random("%(op)s %(batch)d %(new)d" % case)
    total = case["length"] if case["op"] == "attend" else case["cached"] + case["new"]
    out = []
    for b in range(case["batch"]):
        new = case["new"] if b == 0 or case["new"] == 1 else rng.randint((case["new"] + 1) // 2, case["new"])
        cached = total - case["new"]
        out.append((cached if b == 0 else rng.randint(cached // 2, cached), new))
    return out


def _dp(case):
    return (case["head_dim"] + 63) // 64 * 64


# ---------------------------------------------------------------------------------------- inputs
def _positions(case, gen):
    """Position of every token on three axes: text before the visual span, its frames, rows and
    columns, then text that goes on behind the largest of them.  [axes, batch, seq] int32."""
    t, h, w = (int(x) for x in case["grid"].split(","))
    S, B, axes = case["seq"], case["batch"], len(case["sections"].split(","))
    span = t * h * w if t * h * w < S else (S if axes == 2 and t * h * w == S else 0)
    before = min(35, S - span)
    i = torch.arange(S, device=_DEV)
    j = (i - before).clamp(0, max(span - 1, 0))
    grid = torch.stack([j // (h * w), j // w % h, j % w])
    visual = (i >= before) & (i < before + span)
    after = before + max(t, h, w) + i - before - span
    text = torch.where(i < before, i, after)
    pos = torch.where(visual[None], before + grid, text[None].expand(3, S))
    pos = pos[3 - axes:] if axes > 1 else pos[:1]
    shift = torch.randint(0, 64, (1, B, 1), generator=gen, device=_DEV) + case["far"]
    return (pos[:, None] + shift).to(torch.int32).contiguous()


def _rope_state(case, gen):
    B, S, Hq, Hk, dh = (case[n] for n in ("batch", "seq", "q_heads", "kv_heads", "head_dim"))
    dt = _TORCH[case["dtype"]]
    if case["qkv"]:  # views of one [batch, seq, (q + k + v) heads * head_dim] projection
        qkv = torch.randn((B, S, Hq + 2 * Hk, dh), generator=gen, device=_DEV).to(dt)
        q, k = qkv[:, :, :Hq].transpose(1, 2), qkv[:, :, Hq:Hq + Hk].transpose(1, 2)
    else:
        q = torch.randn((B, Hq, S, dh), generator=gen, device=_DEV).to(dt)
        k = torch.randn((B, Hk, S, dh), generator=gen, device=_DEV).to(dt)
    freq = 1e6 ** (-torch.arange(dh // 2, dtype=torch.float64, device=_DEV) * 2 / dh)
    sections = tuple(int(x) for x in case["sections"].split(","))
    shape = SimpleNamespace(dtype=case["dtype"], batch=B, seq_len=S, q_heads=Hq, kv_heads=Hk, head_dim=dh,
                            rot_dim=dh, sections=sections, order=int(case["cycled"]),
                            pairing=int(case["adjacent"]), inverse=int(case["inverse"]))
    return {"shape": shape, "q": q, "k": k, "positions": _positions(case, gen), "inv_freq": freq}


def _cache_shape(case, max_len, dtype="bf16"):
    block = case["block"]
    wide = (max_len + block - 1) // block
    return SimpleNamespace(dtype=case.get("dtype", dtype), batch=case["batch"],
                           q_heads=case.get("q_heads", case.get("kv_heads", 1)),
                           kv_heads=case.get("kv_heads", 1), head_dim=case.get("head_dim", 64),
                           block_size=block, n_blocks=0, max_blocks=wide, n_new=case["new"],
                           max_len=0, scale=0.0)


def _tables(case, lens, wide, gen):
    """A block table for these lengths, blocks in no order, and how many blocks there are."""
    need = torch.tensor([(n + case["block"] - 1) // case["block"] for n in lens], device=_DEV)
    total = int(sum((n + case["block"] - 1) // case["block"] for n in lens))
    order = torch.randperm(total + 3, generator=gen, device=_DEV).to(torch.int32)
    col = torch.arange(wide, device=_DEV)[None]
    index = (need.cumsum(0) - need)[:, None] + col
    return torch.where(col < need[:, None], order[index.clamp(max=total)], -1).contiguous(), total + 3


def _exponent(amax):
    """The least e with amax <= 448 * 2^e, held inside what a scale may be (448 = 0.875 * 2^9)."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(amax > 0, e, _EXP_LO).clamp(_EXP_LO, _EXP_HI)


def _random_cache(case, blocks, gen):
    """Keys and values N(0, 1), quantised with a scale per block and head.  Every value is drawn alike,
    so they are drawn in the cache's own order."""
    H, n16, dp = case["kv_heads"], case["block"] // 16, _dp(case)
    out = {}
    for name, tail in (("k", (dp // 16, 16, 16)), ("v", (dp // 64, 4, 16, 4, 4))):
        data = torch.empty((blocks, H, n16) + tail, dtype=torch.uint8, device=_DEV)
        scale = torch.empty((blocks, H), device=_DEV)
        step = max(1, (1 << 26) // (H * n16 * 16 * dp))
        for a in range(0, blocks, step):
            part = data[a:a + step]
            x = torch.randn(part.shape, generator=gen, device=_DEV)
            # the dims past head_dim are zero
            d = torch.arange(dp, device=_DEV)
            real = (d < case["head_dim"]).view((dp // 16, 1, 16) if name == "k" else (dp // 64, 1, 4, 16, 1))
            x = x * (real if name == "k" else real.transpose(2, 3))
            e = _exponent(x.reshape(part.shape[0], H, -1).abs().amax(-1))
            s = torch.exp2(e.float())
            part.copy_((x / s.view(s.shape + (1,) * (x.dim() - 2))).to(_FP8).view(torch.uint8))
            scale[a:a + step] = s
        out[name], out[name + "_scale"] = data, scale
    return out


def prepare(case, seed):
    gen = torch.Generator(device=_DEV)
    gen.manual_seed(seed)
    if case["op"] == "rope":
        return _rope_state(case, gen)
    lens = _lengths(case)
    int32 = lambda v: torch.tensor(v, dtype=torch.int32, device=_DEV)  # noqa: E731
    cached, new = int32([c for c, _ in lens]), int32([n for _, n in lens])
    longest = max(c + n for c, n in lens)
    shape = _cache_shape(case, longest)
    block = case["block"]
    if case["op"] == "plan":
        table, used = _tables(case, [c for c, _ in lens], shape.max_blocks, gen)
        need = sum((c + n + block - 1) // block - (c + block - 1) // block for c, n in lens)
        shape.n_blocks = used + need + 5
        # the blocks no request holds, in no order; the first two of them have been handed out already
        free = (used + torch.randperm(need + 5, generator=gen, device=_DEV)).to(torch.int32)
        return {"shape": shape, "cached_len": cached, "new_len": new, "free_blocks": free,
                "free_head": int32([2]), "block_table": table}
    table, shape.n_blocks = _tables(case, [c + n for c, n in lens], shape.max_blocks, gen)
    state = {"shape": shape, "cache": _random_cache(case, shape.n_blocks, gen), "new_len": new}
    if case["op"] == "store":
        B, H, S, dh, dt = case["batch"], case["kv_heads"], case["new"], case["head_dim"], _TORCH[case["dtype"]]
        for name in ("k", "v"):
            state[name] = torch.randn((B, H, S, dh), generator=gen, device=_DEV).mul_(1.5).to(dt)
        r = torch.arange(S, device=_DEV)[None]
        p = cached[:, None] + r
        page = table.gather(1, (p // block).clamp(max=shape.max_blocks - 1))
        state["slot_map"] = torch.where(r < new[:, None], page * block + p % block, -1).to(torch.int32)
        return state
    state.update(block_table=table, kv_len=cached + new)
    state["q"] = torch.randn((case["batch"], case["q_heads"], case["new"], case["head_dim"]), generator=gen,
                             device=_DEV).to(_TORCH[case["dtype"]])
    return state


# ----------------------------------------------------------------------------------- plain forms
def _axis_of_pair(shape):
    """Axis of every pair: the sections one after the other, or dealt in turn until each is used up."""
    left, axes = list(shape.sections), []
    if not shape.order:
        return [a for a, n in enumerate(left) for _ in range(n)]
    rounds = [(i, a) for a, n in enumerate(left) for i in range(n)]
    return [a for _, a in sorted(rounds)]


def _rope_plain(s):
    sh = s["shape"]
    axis = torch.tensor(_axis_of_pair(sh), device=_DEV)
    # 64 bits: a far position's angle has few digits behind the point in 32
    angle = s["positions"][axis].double() * s["inv_freq"][:, None, None]
    angle = angle.permute(1, 2, 0)[:, None]
    cos, sin = angle.cos().float(), angle.sin().float()
    if sh.inverse:
        sin = -sin
    half, out = sh.rot_dim // 2, {}
    for name in ("q", "k"):
        x = s[name].float()
        a, b = (x[..., 0::2], x[..., 1::2]) if sh.pairing else (x[..., :half], x[..., half:])
        pair = (a * cos - b * sin, a * sin + b * cos)
        y = torch.stack(pair, -1).flatten(-2) if sh.pairing else torch.cat(pair, -1)
        out[name] = y.to(s[name].dtype).contiguous()
    return out


def _plan_plain(s):
    sh, bs = s["shape"], s["shape"].block_size
    c, n, table, free = s["cached_len"].long(), s["new_len"].long(), s["block_table"], s["free_blocks"]
    first, end = (c + bs - 1) // bs, (c + n + bs - 1) // bs
    need = end - first
    head = s["free_head"].long()
    base = head + need.cumsum(0) - need
    total = need.sum()
    missing = (head + total - free.numel()).clamp(min=0)
    ok = missing == 0
    col = torch.arange(sh.max_blocks, device=_DEV)[None]
    fresh = (col >= first[:, None]) & (col < end[:, None]) & ok
    taken = free[(base[:, None] + col - first[:, None]).clamp(0, free.numel() - 1)]
    table = torch.where(fresh, taken, table)
    r = torch.arange(sh.n_new, device=_DEV)[None]
    p = c[:, None] + r
    page = table.gather(1, (p // bs).clamp(max=sh.max_blocks - 1)).long()
    slot = torch.where((r < n[:, None]) & ok, page * bs + p % bs, -1)
    return {"block_table": table, "slot_map": slot.to(torch.int32),
            "kv_len": torch.where(ok, c + n, c).to(torch.int32),
            "free_head": torch.where(ok, head + total, head).to(torch.int32), "missing": missing.to(torch.int32)}


def _k_rows(data):
    """[..., n16, dp/16, 16, 16] -> [..., tokens, dp]."""
    return data.transpose(-3, -2).flatten(-2).flatten(-3, -2)


def _k_pack(rows):
    """The inverse of _k_rows."""
    return rows.unflatten(-2, (-1, 16)).unflatten(-1, (-1, 16)).transpose(-3, -2).contiguous()


def _v_rows(data):
    """[..., n16, h, g, i, s, r] -> [..., tokens (n16, g, r), dp (h, s, i)]."""
    d = data.dim() - 6
    keep = list(range(d))
    return data.permute(keep + [d, d + 2, d + 5, d + 1, d + 4, d + 3]).flatten(-3).flatten(-4, -2)


def _v_pack(rows):
    x = rows.unflatten(-2, (-1, 4, 4)).unflatten(-1, (-1, 4, 16))  # [..., n16, g, r, h, s, i]
    d = x.dim() - 6
    return x.permute(list(range(d)) + [d, d + 3, d + 1, d + 5, d + 4, d + 2]).contiguous()


def _store_plain(s):
    sh, bs, cache = s["shape"], s["shape"].block_size, s["cache"]
    slot, (B, S) = s["slot_map"].long(), s["slot_map"].shape
    # rows of a sequence by the block that they go to
    runs = (S + bs - 2) // bs + 1
    first = slot[:, :1].clamp(min=0) % bs
    row = torch.arange(runs * bs, device=_DEV)[None] - first
    inside = (row >= 0) & (row < S)
    at = row.clamp(0, S - 1)
    here = slot.gather(1, at)
    valid = (inside & (here >= 0)).view(B, runs, bs)
    page = torch.where(valid, here.view(B, runs, bs) // bs, -1).amax(-1)
    begun = valid[..., 0]                                      # the block's first token is among them
    start = torch.where(valid, torch.arange(bs, device=_DEV), bs).amin(-1)
    b_of, j_of = torch.nonzero(page >= 0, as_tuple=True)
    page, begun, start, valid = page[b_of, j_of], begun[b_of, j_of], start[b_of, j_of], valid[b_of, j_of]
    rows = at.view(B, runs, bs)[b_of, j_of]
    H, dh, dp = sh.kv_heads, sh.head_dim, cache["k"].shape[-3] * 16
    old_rows = (torch.arange(bs, device=_DEV)[None] < start[:, None])[:, None, :, None]
    new_rows = valid[:, None, :, None]
    for name, unpack, pack in (("k", _k_rows, _k_pack), ("v", _v_rows, _v_pack)):
        data, scale = cache[name], cache[name + "_scale"]
        x = s[name][b_of[:, None], :, rows].permute(0, 2, 1, 3).float()          # [pages, H, bs, dh]
        x = torch.where(new_rows, x, 0.0)
        need = torch.exp2(_exponent(x.abs().amax((2, 3))).float())
        before = scale[page]
        after = torch.where(begun[:, None], need, torch.maximum(before, need))
        held = unpack(data[page].view(_FP8).float())                             # [pages, H, bs, dp]
        old = held * (before / after)[..., None, None]
        x = torch.nn.functional.pad(x / after[..., None, None], (0, dp - dh))
        # behind the new tokens: zero in a block that this call begins, as it was in another
        rest = torch.where(begun[:, None, None, None], 0.0, held)
        y = torch.where(new_rows, x, torch.where(old_rows, old, rest))
        data[page] = pack(y.to(_FP8).view(torch.uint8))
        scale[page] = after
    return cache


def _attend_plain(s):
    sh, cache = s["shape"], s["cache"]
    q, (B, Hq, T, dh), H = s["q"], s["q"].shape, sh.kv_heads
    page = s["block_table"].long().clamp(min=0)
    rows = {}
    for name, unpack in (("k", _k_rows), ("v", _v_rows)):
        x = unpack(cache[name][page].view(_FP8).float())                         # [B, W, H, bs, dp]
        x = x * cache[name + "_scale"][page][..., None, None]
        rows[name] = x.transpose(1, 2).flatten(2, 3)[..., :dh]
    L = rows["k"].shape[2]
    logits = q.float().reshape(B, H, Hq // H * T, dh) @ rows["k"].transpose(-1, -2).contiguous()
    logits = logits.view(B, H, Hq // H, T, L) * dh ** -0.5
    t = torch.arange(T, device=_DEV)
    sees = torch.where(t < s["new_len"][:, None], (s["kv_len"] - s["new_len"])[:, None] + t + 1, 0)
    seen = (torch.arange(L, device=_DEV) < sees[..., None])[:, None, None]
    logits = torch.where(seen, logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(logits - torch.where(top == -math.inf, 0.0, top)), 0.0)
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    return (p.view(B, H, -1, L) @ rows["v"].contiguous()).view(B, Hq, T, dh).to(q.dtype)


# ------------------------------------------------------------------------------------------- run
def run(state):
    op = "rope" if "positions" in state else "plan" if "free_blocks" in state else "store" if "slot_map" in state else "attend"
    if own:
        from paper_2505_22654_amd import binding as vb
        sh = state["shape"]
        if op == "rope":
            r = vb.rope(sh, state["positions"], state["inv_freq"], state["q"], state["k"])
            return {"q": r["q"], "k": r["k"]}
        if op == "plan":
            r = vb.cache_plan(sh, state["cached_len"], state["new_len"], state["free_blocks"],
                              state["free_head"], state["block_table"])
            return {n: r[n] for n in ("block_table", "slot_map", "kv_len", "free_head", "missing")}
        if op == "store":
            vb.cache_store(sh, state["k"], state["v"], state["slot_map"], state["cache"])
            return _values(state["cache"])
        return vb.cache_attend(sh, state["q"], state["cache"], state["block_table"], state["kv_len"],
                               state["new_len"])["out"]
    if op == "rope":
        return _rope_plain(state)
    if op == "plan":
        return _plan_plain(state)
    if op == "store":
        return _values(_store_plain(state))
    return _attend_plain(state)


def _values(cache):
    """The 8-bit values as numbers, and the scales."""
    return {n: t if n.endswith("scale") else t.view(_FP8) for n, t in cache.items()}


# ------------------------------------------------------------------------------------------ work
def work(case):
    if case["op"] == "rope":
        es = 4 if case["dtype"] == "f32" else 2
        n = case["batch"] * case["seq"] * (case["q_heads"] + case["kv_heads"]) * case["head_dim"]
        axes = len(case["sections"].split(","))
        return {"bytes": 2 * n * es + 4 * axes * case["batch"] * case["seq"] + 4 * case["head_dim"], "flops": 3 * n}
    lens, bs = _lengths(case), case["block"]
    blocks = sum((c + n + bs - 1) // bs - c // bs for c, n in lens)
    if case["op"] == "plan":
        # lengths in, free blocks in, table entries, slots and lengths out
        return {"bytes": 4 * (3 * case["batch"] + 2 * blocks + case["batch"] * case["new"]), "flops": 0}
    es, H, dh = 4 if case["dtype"] == "f32" else 2, case["kv_heads"], case["head_dim"]
    if case["op"] == "store":
        rows = sum(n for _, n in lens)
        return {"bytes": 2 * rows * H * dh * (es + 1) + 4 * case["batch"] * case["new"] + 2 * 4 * blocks * H,
                "flops": 4 * rows * H * dh}
    held = sum(c + n for c, n in lens)
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in lens)
    pages = sum((c + n + bs - 1) // bs for c, n in lens)
    out = 2 * case["batch"] * case["q_heads"] * case["new"] * dh * es
    return {"bytes": 2 * held * H * dh + 2 * 4 * pages * H + 4 * pages + out,
            "flops": 4 * pairs * case["q_heads"] * dh}


# ----------------------------------------------------------------------------------------- exact
def _e4m3_values():
    """What the 256 codes stand for, from the format: 4 exponent bits with bias 7, 3 mantissa bits."""
    out = []
    for code in range(256):
        e, m = code >> 3 & 15, code & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out.append((-v if code & 128 else v) if code & 127 != 127 else math.nan)
    return torch.tensor(out, dtype=torch.float64, device=_DEV)


def _e4m3_round(y):
    """The nearest e4m3 value, ties to the even one."""
    step = torch.exp2(torch.log2(y.abs().clamp(min=2.0 ** -6)).floor() - 3)
    return torch.round(y / step) * step


def _offset(name, token, dim, dp):
    """Place of a token's value inside its block of one head."""
    if name == "k":
        return token // 16 * 16 * dp + dim // 16 * 256 + token % 16 * 16 + dim % 16
    return (token // 16 * 16 * dp + dim // 64 * 1024 + token % 16 // 4 * 256 + dim % 16 * 16
            + dim % 64 // 16 * 4 + token % 4)


def _exact_rope(s):
    sh = s["shape"]
    turn = s["inv_freq"] * s["positions"].double()[..., None]                    # [axes, B, S, pairs]
    axis = torch.tensor(_axis_of_pair(sh), device=_DEV)
    turn = turn.gather(0, axis.expand((1,) + turn.shape[1:]))[0][:, None]
    z = torch.polar(torch.ones_like(turn), -turn if sh.inverse else turn)
    out = {}
    for name in ("q", "k"):
        x = s[name].double()
        half = sh.rot_dim // 2
        first = torch.arange(half, device=_DEV) * (2 if sh.pairing else 1)
        second = first + (1 if sh.pairing else half)
        w = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * z
        y = torch.empty_like(x)
        y[..., first], y[..., second] = w.real, w.imag
        out[name] = y
    return out


def _exact_store(s):
    sh, bs = s["shape"], s["shape"].block_size
    value, dp, H = _e4m3_values(), s["cache"]["k"].shape[-3] * 16, sh.kv_heads
    token, dim = torch.arange(bs, device=_DEV)[:, None], torch.arange(dp, device=_DEV)[None]
    slots, out = s["slot_map"].tolist(), {}
    for name in ("k", "v"):
        shape = s["cache"][name].shape
        old = value[s["cache"][name].long().flatten()].view(shape[0], H, -1)
        scale = s["cache"][name + "_scale"].double().clone()
        where = _offset(name, token, dim, dp)
        for b, row in enumerate(slots):
            r = 0
            while r < len(row) and row[r] >= 0:
                page, off = row[r] // bs, row[r] % bs
                n = min(bs - off, sum(1 for x in row[r:r + bs - off] if x >= 0))
                x = s[name][b, :, r:r + n].double()
                amax = x.abs().amax((1, 2))
                e = torch.ceil(torch.log2(amax / _MAX)).clamp(_EXP_LO, _EXP_HI)
                need = torch.exp2(e)
                sc = need if off == 0 else torch.maximum(need, scale[page])
                rows = old[page][:, where]
                rows = torch.zeros_like(rows) if off == 0 else rows
                if off:
                    rows[:, :off] = _e4m3_round(rows[:, :off] * (scale[page] / sc)[:, None, None])
                rows[:, off:off + n, :x.shape[-1]] = _e4m3_round(x / sc[:, None, None])
                old[page][:, where] = rows
                scale[page] = sc
                r += n
        out[name], out[name + "_scale"] = old.view(shape), scale
    return out


def _exact_attend(s):
    sh, bs = s["shape"], s["shape"].block_size
    q, H = s["q"].double(), sh.kv_heads
    B, Hq, T, dh = q.shape
    value, dp = _e4m3_values(), s["cache"]["k"].shape[-3] * 16
    out = torch.zeros_like(q)
    lens, new = s["kv_len"].tolist(), s["new_len"].tolist()
    flat = {n: s["cache"][n].view(-1) for n in ("k", "v")}
    dim = torch.arange(dh, device=_DEV)[None]
    for b in range(B):
        j = torch.arange(lens[b], device=_DEV)
        page = s["block_table"][b].long()[j // bs]
        for h in range(H):
            rows = {}
            for n in ("k", "v"):
                at = (page * H + h)[:, None] * bs * dp + _offset(n, (j % bs)[:, None], dim, dp)
                rows[n] = value[flat[n][at].long()] * s["cache"][n + "_scale"].double()[page, h][:, None]
            for g in range(Hq // H):
                i = h * (Hq // H) + g
                x = q[b, i, :new[b]] @ rows["k"].T * dh ** -0.5
                last = lens[b] - new[b] + torch.arange(new[b], device=_DEV)
                x = x.masked_fill(j[None] > last[:, None], -math.inf)
                out[b, i, :new[b]] = torch.softmax(x, -1) @ rows["v"]
    return out


def exact(case, seed):
    if case["op"] == "plan":
        return None
    if case["op"] == "attend" and case["batch"] * case["q_heads"] > 600 and case["length"] > 8000:
        return None
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(s)
    return _exact_store(s) if case["op"] == "store" else _exact_attend(s)
