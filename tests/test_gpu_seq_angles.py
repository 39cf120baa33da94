"""The position rotation against angles reduced exactly."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_1801_04380_amd as sn

pytestmark = pytest.mark.gpu
# 2 pi to 60 places behind the point, from the published digits of pi
TAU = 2 * Fraction(3141592653589793238462643383279502884197169399375105820974944, 10 ** 60)


def exact_turn(position, freq):
    """cos and sin of position * freq: a product of whole numbers and its remainder, in fractions; what is left is below pi."""
    a = Fraction(int(position)) * Fraction(float(freq))
    a -= round(a / TAU) * TAU
    return np.cos(float(a)), np.sin(float(a))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("span", [(0, 1 << 10), ((1 << 24) - 600, 1 << 24), ((1 << 31) - 600, (1 << 31) - 1), (-(1 << 31), -(1 << 31) + 600)])
def test_angles_of_far_positions(span, interleaved):
    """Heads of ones: their mean square is 1 and eps vanishes beside it, so the norm changes nothing and the results are cos - sin and cos + sin.
    Frequencies from 1e-4 to 1000.

    Tolerance: cosine and sine are each within two steps of a value below one, 2^-23; their sum is rounded by half a step below two, 2^-24; the
    root is within a step, 2^-23 of a value up to sqrt 2."""
    Dh = 64
    rng = np.random.RandomState(5)
    pos = np.unique(np.concatenate([[span[0], span[1] - 1], rng.randint(span[0], span[1], 40, dtype=np.int64)]))
    freq = np.concatenate([[1.0, 1000.0, 1e-4], 10 ** rng.uniform(-4, 3, Dh // 2 - 3)]).astype(np.float32)
    x = torch.ones(len(pos), Dh, device="cuda")
    y = torch.empty_like(x)
    sn.sn_headnorm_rot_fwd(x, None, None, None, torch.tensor(pos, dtype=torch.int32, device="cuda"), torch.tensor(freq).cuda(), y, None, Dh, 2.0 ** -30, interleaved)
    y = y.double().cpu().numpy()
    one, two = (y[:, 0::2], y[:, 1::2]) if interleaved else (y[:, :Dh // 2], y[:, Dh // 2:])
    turns = np.array([[exact_turn(p, f) for f in freq] for p in pos])
    c, s = turns[..., 0], turns[..., 1]
    worst = max(np.abs(one - (c - s)).max(), np.abs(two - (c + s)).max())
    assert worst <= 2 * 2.0 ** -23 + 2.0 ** -24 + 2 ** 0.5 * 2.0 ** -23, worst
