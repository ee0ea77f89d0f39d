"""vscan_rope against the definition in 64 bits.

Tolerance, with u = 2^-24 and |x|, |y| the entries of a pair: sine and cosine are off by at most 3 u
(their argument is rounded once, the sums twice), the two products and their sum by 3 u of theirs, so
8 u (|x| + |y|) bounds what precedes the rounding to bf16, which is half a step: 2^-8 of the result."""
import dataclasses
import itertools

import pytest

from paper_2505_22654_amd import binding as vb
from paper_2505_22654_amd import workloads as wl
from tests import decode_reference as ref

pytestmark = pytest.mark.gpu


def _inputs(shape, seed, far=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = vb._torch_dtype(shape.dtype)
    x = {n: torch.randn((shape.batch, h, shape.seq_len, shape.head_dim), generator=g, device="cuda").to(dt)
         for n, h in (("q", shape.q_heads), ("k", shape.kv_heads)) if h}
    pos = torch.randint(-3, 5000, (len(shape.sections), shape.batch, shape.seq_len), generator=g, device="cuda") + far
    return x, pos.to(torch.int32), vb.rope_frequencies(shape.rot_dim, 1e6)


def _check(shape, x, pos, freq, got):
    for n in x:
        want = ref.rope(x[n], pos, freq, shape)
        size = x[n].double()
        if shape.rot_dim:
            r, half = shape.rot_dim, shape.rot_dim // 2
            a, b = (size[..., 0:r:2].abs(), size[..., 1:r:2].abs()) if shape.pairing else (size[..., :half].abs(), size[..., half:r].abs())
            import torch
            pair = torch.stack((a + b, a + b), -1).flatten(-2) if shape.pairing else torch.cat((a + b, a + b), -1)
            pair = torch.cat((pair, torch.zeros_like(size[..., r:])), -1)
        tol = 8 * 2.0 ** -24 * pair + (2.0 ** -8 * want.abs() if shape.dtype == "bf16" else 0)
        worst = ((got[n].double() - want).abs() - tol).max()
        assert float(worst) <= 0, (shape, n, float(worst))
        assert got[n].shape == x[n].shape and got[n].dtype == x[n].dtype


SHAPES = [
    ("bf16", 1, 1, 28, 4, 128, 128, (16, 24, 24)),       # one token
    ("bf16", 3, 77, 7, 1, 128, 128, (16, 24, 24)),
    ("bf16", 2, 33, 4, 4, 72, 72, (18, 18)),             # halves of 36 entries: pieces of 8 bytes
    ("bf16", 2, 19, 2, 2, 80, 40, (20,)),                # the rest of a row is copied
    ("bf16", 1, 5, 3, 0, 8, 8, (1, 2, 1)),               # no keys
    ("bf16", 2, 300, 0, 5, 256, 256, (3, 60, 1, 64)),    # no queries, four axes
    ("bf16", 1, 1000, 33, 2, 64, 24, (12, 0)),           # an axis without pairs
    ("f32", 2, 45, 16, 16, 80, 80, (20, 20)),
    ("f32", 5, 1, 8, 2, 128, 64, (8, 12, 12)),
    ("f32", 1, 129, 1, 1, 104, 104, (52,)),
]


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "-".join(map(str, c[:7])))
@pytest.mark.parametrize("order,pairing,inverse", list(itertools.product((0, 1), (0, 1), (0, 1))))
def test_rope_matches_the_definition(case, order, pairing, inverse):
    shape = wl.RopeShape(*case, order=order, pairing=pairing, inverse=inverse)
    x, pos, freq = _inputs(shape, seed=sum(case[1:7]))
    _check(shape, x, pos, freq, vb.rope(shape, pos, freq, x.get("q"), x.get("k")))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope_at_far_positions(dtype):
    """Angles of positions near the ends of 32 bits keep their digits."""
    shape = wl.RopeShape(dtype, 2, 40, 2, 2, 64, 64, (16, 16))
    x, pos, freq = _inputs(shape, 5, far=2 ** 31 - 6000)
    _check(shape, x, pos, freq, vb.rope(shape, pos, freq, x["q"], x["k"]))
    pos = -pos - 1
    _check(shape, x, pos, freq, vb.rope(shape, pos, freq, x["q"], x["k"]))


@pytest.mark.parametrize("dtype,rot", [("bf16", 64), ("bf16", 24), ("f32", 40)])
@pytest.mark.parametrize("pairing", [0, 1])
def test_rope_strides_and_in_place(dtype, rot, pairing):
    """q and k as views of one projection, turned into new tensors and in place: the same values, and
    nothing else of the projection touched."""
    import torch
    B, S, Hq, Hk, dh = 2, 37, 6, 2, 64
    shape = wl.RopeShape(dtype, B, S, Hq, Hk, dh, rot, (rot // 2 - 3, 3), pairing=pairing)
    qkv = torch.randn((B, S, Hq + 2 * Hk, dh), device="cuda").to(vb._torch_dtype(dtype))
    before = qkv.clone()
    view = lambda t: {"q": t[:, :, :Hq].transpose(1, 2), "k": t[:, :, Hq:Hq + Hk].transpose(1, 2)}  # noqa: E731
    _, pos, freq = _inputs(shape, 9)
    x = view(qkv)
    got = vb.rope(shape, pos, freq, x["q"], x["k"])
    assert torch.equal(qkv, before) and got["q"].is_contiguous()
    _check(shape, x, pos, freq, got)
    same = vb.rope(shape, pos, freq, x["q"].contiguous(), x["k"].contiguous(), out={"q": torch.empty_like(got["q"])})
    vb.rope(shape, pos, freq, x["q"], x["k"], in_place=True)
    for n in "qk":
        assert torch.equal(x[n], got[n]) and torch.equal(same[n], got[n])
    assert torch.equal(qkv[:, :, Hq + Hk:], before[:, :, Hq + Hk:])
    # one row for every sequence can be read, but not turned in place
    k = before[:1, :, Hq:Hq + Hk].transpose(1, 2).expand(B, Hk, S, dh)
    _check(shape, {"k": k}, pos, freq, {"k": vb.rope(shape, pos, freq, x["q"], k)["k"]})
    with pytest.raises(vb.VscanError):
        vb.rope(shape, pos, freq, x["q"], k, in_place=True)
    odd = torch.empty((B, Hk, S, dh + 2), device="cuda").to(k.dtype)[..., :dh]
    with pytest.raises(vb.VscanError):
        vb.rope(shape, pos, freq, x["q"], odd)


@pytest.mark.parametrize("order,pairing", [(0, 0), (1, 1)])
def test_rope_inverse_is_the_gradient(order, pairing):
    """<g, R(x + d) - R(x - d)> / 2 = <R^-1 g, d>: the rotation is linear, so the difference is exact up
    to rounding (128 products of fp32 values, 10 u each)."""
    import torch
    shape = wl.RopeShape("f32", 2, 21, 3, 1, 64, 64, (10, 12, 10), order=order, pairing=pairing)
    x, pos, freq = _inputs(shape, 31)
    back = dataclasses.replace(shape, inverse=1)
    for n, h in (("q", 3), ("k", 1)):
        one = dataclasses.replace(shape, **{"q_heads": h if n == "q" else 0, "kv_heads": h if n == "k" else 0})
        run = lambda t, s: vb.rope(s, pos, freq, **{n: t})[n].double()  # noqa: E731
        g, d = torch.randn_like(x[n]), torch.randn_like(x[n])
        plus, minus = (x[n].double() + d.double()).float(), (x[n].double() - d.double()).float()
        lhs = (g.double() * (run(plus, one) - run(minus, one)) / 2).sum()
        grad = run(g, dataclasses.replace(back, q_heads=one.q_heads, kv_heads=one.kv_heads))
        rhs = (grad * (plus.double() - minus.double()) / 2).sum()
        slack = 10 * 2.0 ** -24 * 2 * (g.double().abs() * (plus.double().abs() + minus.double().abs())).sum() * 2
        assert abs(float(lhs - rhs)) <= float(slack)
        # and it undoes the rotation
        again = vb.rope(dataclasses.replace(back, q_heads=one.q_heads, kv_heads=one.kv_heads), pos, freq,
                        **{n: vb.rope(one, pos, freq, **{n: x[n]})[n]})[n]
        assert float((again - x[n]).abs().max()) <= 2 * 8 * 2.0 ** -24 * 4 * float(x[n].abs().max())


def test_rope_on_another_stream():
    import torch
    shape = wl.RopeShape("bf16", 2, 50, 4, 2, 64, 64, (32,))
    x, pos, freq = _inputs(shape, 3)
    want = vb.rope(shape, pos, freq, x["q"], x["k"])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = vb.rope(shape, pos, freq, x["q"], x["k"])
    s.synchronize()
    assert torch.equal(got["q"], want["q"]) and torch.equal(got["k"], want["k"])


@pytest.mark.parametrize("dtype,dh,extra", [("bf16", 128, 0), ("bf16", 128, 8), ("f32", 64, 0), ("bf16", 72, 0)])
@pytest.mark.parametrize("pairing", [0, 1])
def test_rope_of_more_than_the_caches_hold(dtype, dh, extra, pairing):
    """Tens of megabytes, whole lines and parts of them, into new tensors and in place."""
    import torch
    B, S, Hq, Hk = 3, (36 << 20) // (3 * 32 * dh * (2 if dtype == "bf16" else 4)), 28, 4
    shape = wl.RopeShape(dtype, B, S, Hq, Hk, dh, dh, (dh // 2,), pairing=pairing)
    qkv = torch.randn((B, S, (Hq + Hk) * dh + extra), device="cuda").to(vb._torch_dtype(dtype))
    rows = qkv[..., :(Hq + Hk) * dh].unflatten(2, (Hq + Hk, dh)).transpose(1, 2)
    x = {"q": rows[:, :Hq], "k": rows[:, Hq:]}
    _, pos, freq = _inputs(shape, 4)
    got = vb.rope(shape, pos, freq, x["q"], x["k"])
    _check(shape, x, pos, freq, got)
    vb.rope(shape, pos, freq, x["q"], x["k"], in_place=True)
    assert torch.equal(x["q"], got["q"]) and torch.equal(x["k"], got["k"])


def test_rope_of_rows_more_than_32_bits_apart():
    """Two sequences at either end of 5 GB, read, and turned in place."""
    import torch
    shape = wl.RopeShape("bf16", 2, 9, 3, 2, 128, 128, (64,))
    x, pos, freq = _inputs(shape, 8)
    want = vb.rope(shape, pos, freq, x["q"], x["k"])
    far = torch.empty(5 * (1 << 29) + (1 << 16), dtype=torch.bfloat16, device="cuda")
    y = {n: far[at:].as_strided(t.shape, (5 * (1 << 29),) + t.stride()[1:]) for at, (n, t) in zip((0, 1 << 15), x.items())}
    for n in y:
        y[n].copy_(x[n])
    got = vb.rope(shape, pos, freq, y["q"], y["k"])
    assert torch.equal(got["q"], want["q"]) and torch.equal(got["k"], want["k"])
    vb.rope(shape, pos, freq, y["q"], y["k"], in_place=True)
    assert torch.equal(y["q"], want["q"]) and torch.equal(y["k"], want["k"])
