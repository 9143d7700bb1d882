"""Layer norm where every operand's rows start on 16-byte boundaries, so that the calls take their wide accesses, against 64-bit
formulas: widths up to the longest row that is held in registers, and rows enough for every CTA to go round its ring of rows
several times.  Bounds as in test_gpu_operators."""
import pytest
import torch

from paper_2606_23087_b200 import binding as fp
from test_gpu_operators import B, EPS, U, code, gen, norm_bounds, pool, randn, stream, strided, within  # noqa: F401

pytestmark = pytest.mark.gpu


def forward(pool, rows, cols, dtype):
    g = gen(rows * 10007 + cols)
    x = (randn(g, rows, cols) * torch.exp(randn(g, rows, 1)) + randn(g, rows, 1)).to(dtype)
    w, b = 1 + 0.1 * randn(g, cols), 0.1 * randn(g, cols)
    ldx, ldy = cols + 16, cols + 8
    xs, y = strided(x, ldx), strided(torch.zeros_like(x), ldy)
    assert all(t.data_ptr() % 16 == 0 and t.stride(0) * t.element_size() % 16 == 0 for t in (xs, y)) and cols * x.element_size() % 16 == 0
    mean, rstd = torch.full((2, rows), float("nan"), device="cuda")
    assert pool.layer_norm(rows, cols, xs.data_ptr(), ldx, code(dtype), w.data_ptr(), b.data_ptr(), fp.FT_F32, EPS, y.data_ptr(), ldy,
                           mean.data_ptr(), rstd.data_ptr(), stream()) == 0
    x6, w6, b6 = x.double(), w.double(), b.double()
    m6 = x6.mean(1, keepdim=True)
    r6 = (((x6 - m6) ** 2).mean(1, keepdim=True) + EPS) ** -0.5
    e6 = (x6 - m6) * r6 * w6 + b6
    near = 64 * U * x6.abs().mean(1, keepdim=True)
    within(mean[:, None], m6, near + 1e-30, "mean")
    within(rstd[:, None], r6, r6 * (80 * U + near * r6 + (near * r6) ** 2), "rstd")
    bound = norm_bounds(x6, w6, b6, m6, r6)
    within(y, e6, bound + (B * (e6.abs() + bound) if dtype == torch.bfloat16 else 2 * U * e6.abs()) + 1e-30, "y")
    assert torch.as_strided(y, (rows, 8), (ldy, 1), cols).isnan().all()


# 12288 fp32 columns are the last that 384 threads hold, 16384 the last of either type that registers hold at all
@pytest.mark.parametrize("rows", [1, 5, 700])
@pytest.mark.parametrize("dtype, cols", [(torch.float32, 12288), (torch.float32, 12292), (torch.float32, 14336), (torch.float32, 16384),
                                         (torch.float32, 16388), (torch.bfloat16, 12296), (torch.bfloat16, 16384), (torch.bfloat16, 16392)])
def test_long_rows(pool, rows, cols, dtype):  # noqa: F811
    forward(pool, rows, cols, dtype)
