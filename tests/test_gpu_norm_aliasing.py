"""Norms whose output lies where an input does: with that one's stride they work in place, with another they are refused, because a row would land on
rows that are still to be read."""
import pytest
import torch

from paper_2606_23087_b200 import binding as fp
from test_gpu_more_operators import EPS, INVALID, bits, gen, pool, randn, stream  # noqa: F401

pytestmark = pytest.mark.gpu
ROWS, COLS = 5, 96


def matrix(g, ld):
    return randn(g, ROWS, ld)[:, :COLS]


@pytest.mark.parametrize("rows", [1, ROWS])
def test_rms_norm_on_its_inputs(pool, rows):  # noqa: F811
    g = gen(1)
    w = randn(g, COLS)

    def call(x, res, total, y, ldt, ldy):
        return pool.rms_norm(rows, COLS, x.data_ptr(), x.stride(0), res.data_ptr(), res.stride(0), fp.FT_F32, w.data_ptr(), fp.FT_F32, EPS,
                             0 if total is None else total.data_ptr(), ldt, 0 if y is None else y.data_ptr(), ldy, stream=stream())
    x, res = matrix(g, 128), matrix(g, 128)
    total, y = torch.empty(ROWS, COLS, device="cuda"), torch.empty(ROWS, COLS, device="cuda")
    assert call(x, res, total, y, COLS, COLS) == 0
    want = 0 if rows == 1 else INVALID
    for where in (x, res):
        for ld in (COLS, 100, 128):
            buf_x, buf_r = torch.zeros(ROWS, 128, device="cuda"), torch.zeros(ROWS, 128, device="cuda")
            buf_x[:, :COLS], buf_r[:, :COLS] = x, res
            x2, res2 = buf_x[:, :COLS], buf_r[:, :COLS]
            at = x2 if where is x else res2
            assert call(x2, res2, at, None, ld, 0) == (0 if ld == 128 else want), ld
            if ld == 128 or rows == 1:
                assert torch.equal(bits(at[:rows]), bits(total[:rows]))
                at.copy_(where)
            assert call(x2, res2, None, at, 0, ld) == (0 if ld == 128 else want), ld
            if ld == 128 or rows == 1:
                assert torch.equal(bits(at[:rows]), bits(y[:rows]))
    assert call(x, res, total, total, COLS, COLS) == INVALID


@pytest.mark.parametrize("rows", [1, ROWS])
def test_rms_norm_grad_on_its_inputs(pool, rows):  # noqa: F811
    g = gen(2)
    w, rstd = randn(g, COLS), torch.rand(ROWS, device="cuda", generator=g) + 0.5
    n = pool.rms_norm_grad_workspace(ROWS, COLS)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    values = [matrix(g, 128) for _ in range(3)]

    def call(m, dx, ld):
        dy, s, dsum = m
        return pool.rms_norm_grad(rows, COLS, dy.data_ptr(), dy.stride(0), s.data_ptr(), s.stride(0), dsum.data_ptr(), dsum.stride(0), fp.FT_F32, w.data_ptr(), fp.FT_F32,
                                  rstd.data_ptr(), dx.data_ptr(), ld, 0, False, ws.data_ptr(), n, stream())
    exp = torch.empty(ROWS, COLS, device="cuda")
    assert call(values, exp, COLS) == 0
    for which in range(3):
        for ld in (COLS, 100, 128):
            m = []
            for v in values:
                b = torch.zeros(ROWS, 128, device="cuda")
                b[:, :COLS] = v
                m.append(b[:, :COLS])
            ok = ld == 128 or rows == 1
            assert call(m, m[which], ld) == (0 if ok else INVALID), (which, ld)
            assert torch.equal(bits(m[which][:rows]), bits((exp if ok else values[which])[:rows]))


@pytest.mark.parametrize("rows", [1, ROWS])
def test_layer_norm_on_its_inputs(pool, rows):  # noqa: F811
    g = gen(3)
    w, mean, rstd = randn(g, COLS), randn(g, ROWS), torch.rand(ROWS, device="cuda", generator=g) + 0.5
    n = pool.layer_norm_grad_workspace(ROWS, COLS)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    values = [matrix(g, 128) for _ in range(2)]

    def norm(m, y, ld):
        return pool.layer_norm(rows, COLS, m[0].data_ptr(), m[0].stride(0), fp.FT_F32, w.data_ptr(), 0, fp.FT_F32, EPS, y.data_ptr(), ld, stream=stream())

    def grad(m, dx, ld):
        return pool.layer_norm_grad(rows, COLS, m[1].data_ptr(), m[1].stride(0), m[0].data_ptr(), m[0].stride(0), fp.FT_F32, w.data_ptr(), fp.FT_F32, mean.data_ptr(),
                                    rstd.data_ptr(), dx.data_ptr(), ld, 0, 0, False, ws.data_ptr(), n, stream())
    for call, on in ((norm, (0,)), (grad, (0, 1))):
        exp = torch.empty(ROWS, COLS, device="cuda")
        assert call(values, exp, COLS) == 0
        for which in on:
            for ld in (COLS, 100, 128):
                m = []
                for v in values:
                    b = torch.zeros(ROWS, 128, device="cuda")
                    b[:, :COLS] = v
                    m.append(b[:, :COLS])
                ok = ld == 128 or rows == 1
                assert call(m, m[which], ld) == (0 if ok else INVALID), (which, ld)
                assert torch.equal(bits(m[which][:rows]), bits((exp if ok else values[which])[:rows]))
