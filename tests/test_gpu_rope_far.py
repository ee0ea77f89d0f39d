"""vscan_rope's sines and cosines against those of the exact angle, reduced in integers, over all of int32.

Tolerance, with u = 2^-24: the rest of the angle, at most pi/4, is rounded once (0.79 u), and its square, the sums
and the product of the sine's again (the last sum half a unit of a value of at most 1, 0.5 u; what it adds has
at most a third of that value, with 3 roundings of u each, 1 u; the Taylor remainder 0.03 u): 3 u."""
from fractions import Fraction

import numpy as np
import pytest

from paper_2505_22654_amd import binding as vb
from paper_2505_22654_amd import workloads as wl

pytestmark = pytest.mark.gpu
PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def _exact(position, freq):
    """(cos, sin) of position * freq, as doubles of the reduced angle."""
    w = Fraction(int(position)) * Fraction(float(freq))
    turns = w / (2 * PI)
    w -= 2 * PI * round(turns)
    return np.cos(float(w)), np.sin(float(w))


@pytest.mark.parametrize("inverse", [0, 1])
@pytest.mark.parametrize("theta", [1e4, 3.7, 1e7])
def test_angles_of_far_positions_are_those_of_the_exact_product(theta, inverse):
    import torch
    rng = np.random.default_rng(int(theta))
    ends = [2 ** 31 - 1, -2 ** 31, -2 ** 31 + 1, 2 ** 30, -2 ** 30 - 1, 0, 1, -1, 355, 710, 103993, 1073741824 - 7]
    near = rng.integers(2 ** 31 - 10 ** 6, 2 ** 31, 60).tolist()
    any_ = rng.integers(-2 ** 31, 2 ** 31, 60).tolist()
    small = (2.0 ** rng.uniform(0, 31, 60)).astype(np.int64).tolist()
    pos = [max(-2 ** 31, min(2 ** 31 - 1, int(p))) for p in ends + near + any_ + small]
    S, rot = len(pos), 32
    shape = wl.RopeShape("f32", 1, S, 1, 0, rot, rot, (rot // 2,), inverse=inverse)
    freq = vb.rope_frequencies(rot, theta)
    freq[3] = 1.0
    freq[5] = 1.25
    x = torch.zeros((1, 1, S, rot), device="cuda")
    x[..., :rot // 2] = 1.0                                          # (1, 0) becomes (cos w, sin w)
    got = vb.rope(shape, torch.tensor(pos, dtype=torch.int64, device="cuda").to(torch.int32).view(1, 1, S), freq, x)["q"].double().cpu().numpy()[0, 0]
    f = freq.cpu().numpy()
    want = np.array([[_exact(p, w) for w in f] for p in pos])        # [S, pairs, 2]
    sign = -1.0 if inverse else 1.0
    off = np.maximum(np.abs(got[:, :rot // 2] - want[..., 0]), np.abs(got[:, rot // 2:] - sign * want[..., 1]))
    worst = np.unravel_index(off.argmax(), off.shape)
    assert off.max() <= 3 * 2.0 ** -24, (pos[worst[0]], f[worst[1]], off.max() * 2.0 ** 24)
