"""The token loss where logits overflow.  Helpers and bounds are test_gpu_operators'."""
import pytest
import torch

from test_gpu_operators import B, U, gen, pool, randn, run_loss, within  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_label_whose_logit_is_minus_infinity(pool):  # noqa: F811
    """The label's logit overflows to -inf (two rows; in one of them another word's does too): its probability is 0, so the loss is
    infinite, lse is that of the other words, and the gradients are finite."""
    hidden, vocab, rows = 64, 700, 5
    g = gen(9)
    w = (randn(g, vocab, hidden) * 0.125).bfloat16()
    w[:, 0] = 0
    w[3, 0] = w[650, 0] = -1e30
    x = randn(g, rows, hidden).bfloat16()
    x[:, 0] = 0
    x[1, 0] = x[4, 0] = 1e30
    labels = torch.tensor([5, 3, 3, 699, 650], device="cuda", dtype=torch.int32)
    z = x.double() @ w.double().T
    z = torch.where(z < -3.4e38, -torch.inf, z)
    lse = torch.logsumexp(z, 1)
    tz = 2 * U * (hidden + 8) * torch.where(z.isfinite(), x.double().abs() @ w.double().abs().T, 0.0).amax(1)
    d = torch.exp(z - lse[:, None])
    d[torch.arange(rows, device="cuda"), labels.long()] -= 1
    dw = torch.full((vocab, hidden), float("nan"), device="cuda")
    for out in (run_loss(pool, x, w, labels), run_loss(pool, x, w, labels, dw=dw)):
        rc, loss, got, dx = out
        assert rc == 0
        within(got, lse, tz + (32 + 0.02 * vocab) * U + 4 * U * (lse.abs() + 16), "lse")
        assert loss[[1, 4]].isposinf().all() and loss[[0, 2, 3]].isfinite().all()
    assert dx.isfinite().all() and dw.isfinite().all()
    # the columns in which nothing is large: d is off by 4 roundings to bf16 (see loss_formula) and the logits' errors
    t = d.abs() * (4 * B + 4 * float(tz.max())) + 1e-30
    x6, w6 = x.double()[:, 1:], w.double()[:, 1:]
    within(dw[:, 1:], d.T @ x6, t.T @ x6.abs() + 2 * U * 64 * (d.abs().T @ x6.abs()), "dw")
    within(dx[:, 1:], d @ w6, t @ w6.abs() + 2 * U * (vocab + 64) * (d.abs() @ w6.abs()) + 1.01 * B * (d @ w6).abs(), "dx")
