"""Rotary positions at the ends of their range against integer arithmetic: the angle in turns is off by less than 2^-31 and rounded to fp32 by up to
2^-26."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2606_23087_b200 import binding as fp
from test_gpu_more_operators import pool, stream  # noqa: F401

pytestmark = pytest.mark.gpu
PI = Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49)


def turns(position, freq):
    """The angle's fraction of a turn, from -1/2 on, to 1e-19: what is left of pi's 50 digits at 2^31 x 8 radians."""
    t = Fraction(freq) * position / (2 * PI)
    return float(t - math.floor(t + Fraction(1, 2)))


@pytest.mark.parametrize("inverse", [False, True])
def test_far_positions(pool, inverse):  # noqa: F811
    rng = np.random.default_rng(5)
    freqs = np.concatenate([[8.0, -8.0, 2 * math.pi, math.pi, 1.0, 1e-4, 1e-9, 0.0, np.nextafter(8.0, 0)], rng.uniform(-8, 8, 55)])
    positions = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, 10 ** 6, -10 ** 9] + [int(v) for v in rng.integers(-2 ** 31, 2 ** 31, 24)]
    n, rows = len(freqs), len(positions)
    pos = torch.tensor([positions], dtype=torch.int32, device="cuda")
    x = torch.zeros(rows, 2 * n, device="cuda")
    x[:, :n] = 1   # (1, 0) turns into (cos, sin)
    t = [fp.RotaryTensor(src=x.data_ptr(), dst=x.data_ptr(), src_row=2 * n, src_head=2 * n, dst_row=2 * n, dst_head=2 * n, heads=1, dtype=fp.FT_F32)]
    assert pool.rotary(rows, pos.data_ptr(), rows, fp.rotary_config(freqs, None, 2 * n, inverse=inverse), t, stream()) == 0
    angle = torch.tensor([[2 * math.pi * turns(p, f) for f in freqs] for p in positions], dtype=torch.float64) * (-1 if inverse else 1)
    bound = 2 * math.pi * (2.0 ** -31 + 2.0 ** -26) + 4 * 2.0 ** -24   # and 2 ulp of a sine below one
    assert float((x[:, :n].double().cpu() - angle.cos()).abs().max()) <= bound
    assert float((x[:, n:].double().cpu() - angle.sin()).abs().max()) <= bound
