"""AdamW where second moments or eps are near the end of fp32's range.  Helpers and bounds are test_gpu_operators'."""
import pytest
import torch

from paper_2606_23087_b200 import binding as fp
from test_gpu_operators import CFG, U, AdamwCase, pool, stream, within  # noqa: F401

pytestmark = pytest.mark.gpu


def first_step(pool, bits, eps, empty):  # noqa: F811
    """One block's gradients go from 1e8 down to 1e-20, whose square is a subnormal number: the first step is lr times the gradient's
    sign all the same, and zero where there is no gradient (every third element of the last block, with `empty`)."""
    n = 256 * 3
    c = AdamwCase(4, n, torch.float32, torch.float32, bits, False, zero=True)
    g = torch.randn(n, generator=torch.Generator().manual_seed(5)).sign() * 10.0 ** torch.linspace(-20, 8, 256).repeat(3)
    if empty:
        g[512::3] = 0
    c.g, c.wd = g, 0.0
    c.dev[1][1].copy_(g.view(torch.uint8).cuda())
    p0 = c.p.double()
    assert pool.adamw_step([c.tensor()], fp.AdamwConfig(**{**CFG, "eps": eps}, step=1), stream()) == 0
    torch.cuda.synchronize()
    f = lambda v: torch.tensor(v, dtype=torch.float64).float()  # noqa: E731
    m, v = f(1 - CFG["beta1"]) * g, f(1 - CFG["beta2"]) * (g * g)
    step = torch.where(g != 0, CFG["lr"] / (1 - CFG["beta1"]) * m.double() / (v.sqrt().double() / (1 - CFG["beta2"]) ** 0.5 + eps), 0.0)
    assert step.isfinite().all()
    within(c.host(0), p0 - step, 16 * U * step.abs() + 8 * U * p0.abs() + 1e-37, "parameters")


@pytest.mark.parametrize("bits", [32, 8])
def test_second_moments_below_the_normal_numbers(pool, bits):  # noqa: F811
    first_step(pool, bits, 0.0, False)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-42, 1e-50])
def test_an_epsilon_below_the_normal_numbers(pool, bits, eps):  # noqa: F811
    first_step(pool, bits, eps, True)
