"""Plain 64-bit statements of the operators around the pruned prefill, from their definitions, with
explicit index arithmetic (torch on any device; nothing here calls the library)."""
import math

import torch

EXP_LO, EXP_HI = -120, 120


def e4m3_values(device="cpu"):
    """What the 256 codes stand for: 4 exponent bits of bias 7, 3 mantissa bits, no infinity."""
    out = []
    for code in range(256):
        e, m = code >> 3 & 15, code & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out.append(math.nan if code & 127 == 127 else -v if code & 128 else v)
    return torch.tensor(out, dtype=torch.float64, device=device)


def e4m3_round(y):
    """Nearest e4m3 value, ties to even, of numbers of at most 448."""
    step = torch.exp2(torch.log2(y.abs().clamp(min=2.0 ** -6)).floor() - 3)
    return torch.round(y / step) * step


def scale_of(amax):
    """Least power of two s with amax <= 448 s."""
    if amax == 0:
        return 2.0 ** EXP_LO
    m, e = math.frexp(amax / 448.0)
    return 2.0 ** min(max(e - 1 if m == 0.5 else e, EXP_LO), EXP_HI)


def offset(kind, token, dim, dp):
    """Place of (token, dim) inside a block of one head."""
    if kind == "k":
        return token // 16 * 16 * dp + dim // 16 * 256 + token % 16 * 16 + dim % 16
    return (token // 16 * 16 * dp + dim // 64 * 1024 + token % 16 // 4 * 256 + dim % 16 * 16
            + dim % 64 // 16 * 4 + token % 4)


def axis_of_pair(sections, order):
    if order == 0:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    left, out = list(sections), []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                left[a] -= 1
                out.append(a)
    return out


def rope(x, positions, inv_freq, shape):
    """x [B,H,S,dh] turned, in 64 bits."""
    x, half = x.double().clone(), shape.rot_dim // 2
    y = x.clone()
    for i, a in enumerate(axis_of_pair(shape.sections, shape.order)):
        u, v = (2 * i, 2 * i + 1) if shape.pairing else (i, half + i)
        w = (positions[a].double() * inv_freq[i].double())[:, None]
        c, s = w.cos(), w.sin() * (-1 if shape.inverse else 1)
        y[..., u] = x[..., u] * c - x[..., v] * s
        y[..., v] = x[..., u] * s + x[..., v] * c
    return y


def plan(shape, cached, new, free, head, table):
    """Lists in; (table, slot_map, kv_len, head, missing) as lists out."""
    bs, cap = shape.block_size, shape.max_blocks * shape.block_size
    head = min(max(head, 0), len(free))
    held = []
    for c, n in zip(cached, new):
        c = min(max(c, 0), cap)
        held.append((c, min(max(n, 0), shape.n_new, cap - c)))
    need = [-(-(c + n) // bs) - -(-c // bs) for c, n in held]
    missing = max(0, head + sum(need) - len(free))
    table = [list(r) for r in table]
    slots, kv_len = [], []
    for b, (c, n) in enumerate(held):
        if missing:
            slots.append([-1] * shape.n_new)
            kv_len.append(c)
            continue
        for j in range(-(-c // bs), -(-(c + n) // bs)):
            table[b][j] = free[head]
            head += 1
        row = []
        for r in range(shape.n_new):
            block = table[b][(c + r) // bs] if r < n else -1
            row.append(block * bs + (c + r) % bs if 0 <= block < shape.n_blocks else -1)
        slots.append(row)
        kv_len.append(c + n)
    return table, slots, kv_len, head, missing


def read(cache, shape, kind):
    """Values [n_blocks, Hkv, block_size, dp] of a cache, without their scales."""
    bs, dp = shape.block_size, (shape.head_dim + 63) // 64 * 64
    data = cache[kind]
    t, d = torch.arange(bs, device=data.device)[:, None], torch.arange(dp, device=data.device)[None]
    return e4m3_values(data.device)[data.reshape(shape.n_blocks, shape.kv_heads, -1).long()][:, :, offset(kind, t, d, dp)]


def codes(values, shape, kind):
    """The bytes of a cache that hold `values` (numbers of the format), the inverse of `read`."""
    bs, dp = shape.block_size, (shape.head_dim + 63) // 64 * 64
    dev = values.device
    table = e4m3_values(dev)
    # code by magnitude; the sign bit on top (a negative zero does not come up)
    mag = torch.searchsorted(table[:127].contiguous(), values.abs().contiguous())
    byte = (mag + 128 * (values < 0)).to(torch.uint8)
    t, d = torch.arange(bs, device=dev)[:, None], torch.arange(dp, device=dev)[None]
    out = torch.zeros(values.shape[:2] + (bs * dp,), dtype=torch.uint8, device=dev)
    out[:, :, offset(kind, t, d, dp)] = byte
    return out


def store(shape, x, slot_map, values, scales):
    """Rows x [B,Hkv,T,dh] into `values` [n_blocks,Hkv,bs,dp] and `scales` [n_blocks,Hkv], in place."""
    bs = shape.block_size
    for b, slots in enumerate(slot_map.tolist()):
        r = 0
        while r < len(slots):
            block, off = slots[r] // bs, slots[r] % bs
            if slots[r] < 0 or block >= shape.n_blocks:
                break
            n = 1
            while n < bs - off and r + n < len(slots) and slots[r + n] == slots[r] + n:
                n += 1
            for h in range(shape.kv_heads):
                rows = x[b, h, r:r + n].double()
                need, old = scale_of(float(rows.abs().max())), float(scales[block, h])
                s = need if off == 0 else max(need, old)
                if off == 0:
                    values[block, h] = 0
                elif s > old:
                    values[block, h, :off] = e4m3_round(values[block, h, :off] * (old / s))
                values[block, h, off:off + n] = 0
                values[block, h, off:off + n, :x.shape[3]] = e4m3_round(rows / s)
                scales[block, h] = s
            r += n


def attend(shape, q, k_rows, v_rows, v_scales, table, kv_len, new_len):
    """(out, bound) in 64 bits.  k_rows, v_rows: values with scales, [n_blocks,Hkv,bs,dh]; v_scales
    [n_blocks,Hkv].  `bound` is what rounding may move a result by, apart from the last one: with u =
    2^-24 a logit of dh products is off by at most (dh + 8) u sum|q k| scale (the products are exact; in
    bf16 calls an entry of q below 2^-13 of its row's largest may be off by 2^-21 of that, as two e4m3
    planes hold multiples of 2^-13 under a scale that puts the largest at 2^7 or more),
    a weight by that twice and the exponential's 4 u, the two sums by (keys + 64) u.  Then the weights'
    rounding.  fp32: three planes of 8 bits, 2^-26 of a weight.  bf16 calls: fp16, half a step of
    which is 2^-11 of a weight, or below fp16's normal numbers 2^-25.  A value's scale s goes with the value
    down to 2^-15 of the largest scale S, beyond that with the weight, so a weight's error of 2^-25 moves a sum
    by at most 2^-25 448 S; and the reference is such that the largest p_j min(1, 2^15 s_j / S) of a wave's keys
    is 2^4 or more.  Divided by that: 2^-29 448 S max_j(p_j min(1, 2^15 s_j / S)) a key.  (A wave whose own largest
    scale is t < S: 2^-29 448 t max_j(p_j min(1, 2^15 s_j / t)), which is less, as t min(1, 2^15 s_j / t) =
    min(t, 2^15 s_j) grows with t.)"""
    bs, T, G = shape.block_size, shape.n_new, shape.q_heads // shape.kv_heads
    dh, u = shape.head_dim, 2.0 ** -24
    scale = shape.scale if shape.scale > 0 else dh ** -0.5
    cap = shape.max_len or shape.max_blocks * bs
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    planes, floor = (2.0 ** -11, 448 * 2.0 ** -29) if shape.dtype == "bf16" else (2.0 ** -26, 0.0)
    for b in range(shape.batch):
        n = T if new_len is None else min(max(int(new_len[b]), 0), T)
        length = min(max(int(kv_len[b]), 0), cap)
        if n == 0 or length == 0:
            continue
        j = torch.arange(length, device=q.device)
        block = table[b].long()[j // bs]
        there = (block >= 0) & (block < shape.n_blocks)
        block = block.clamp(0, shape.n_blocks - 1)
        pos = length - n + torch.arange(n, device=q.device)
        seen = (j[None] <= pos[:, None]) & there[None]
        for h in range(shape.q_heads):
            # (what is not seen may hold anything)
            k = torch.where(there[:, None], k_rows[block, h // G, j % bs], 0.0)
            v = torch.where(there[:, None], v_rows[block, h // G, j % bs], 0.0)
            x = q[b, h, :n].double()
            logits = (x @ k.T * scale).masked_fill(~seen, -math.inf)
            off = (x.abs() @ k.abs().T * scale).masked_fill(~seen, 0.0).amax(1, keepdim=True) * (dh + 8) * u
            if shape.dtype == "bf16":
                top = x.abs().nan_to_num(0).amax(1, keepdim=True)
                small = (x.abs() < 2.0 ** -13 * top) * top * 2.0 ** -21
                off = off + (small @ k.abs().T * scale).masked_fill(~seen, 0.0).amax(1, keepdim=True)
            p = torch.where(seen.any(1, keepdim=True), torch.softmax(logits, 1), 0.0)
            out[b, h, :n] = p @ v
            s = torch.where(there, v_scales.double()[block, h // G], 0.0)
            bound[b, h, :n] = ((p @ v.abs()) * (2 * off + (length + 72) * u + planes)
                               + length * floor * (p * torch.minimum(s.amax(), 2.0 ** 15 * s)).amax(1, keepdim=True))
    return out, bound
