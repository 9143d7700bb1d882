"""The gradient of a log probability at a temperature, by the token loss of scaled rows, against autograd in 64 bits."""
import pytest
import torch

from paper_2606_23087_b200 import binding as fp
from test_gpu_logprobs_precision import inputs
from test_gpu_more_operators import pool, run_scores, stream  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [0.5, 1.0, 4.0])
def test_gradient_at_a_temperature(pool, scale):  # noqa: F811
    rows, hidden, vocab = 40, 256, 1000
    x, w, tokens = inputs(4, rows, hidden, vocab, False)
    x64, w64 = x.double().requires_grad_(), w.double().requires_grad_()
    weight = torch.linspace(-1, 1, rows, device="cuda")
    logp = torch.log_softmax(scale * x64 @ w64.T, 1).gather(1, tokens.long()[:, None])[:, 0]
    (logp * weight.double()).sum().backward()
    xs = (x.float() * scale).bfloat16()
    assert torch.equal(xs.float(), x.float() * scale)
    grad, loss, lse = -weight, torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty(vocab, hidden, device="cuda")
    n = pool.token_loss_workspace(rows, hidden, vocab, True)[1]
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    assert pool.token_loss_grad(rows, hidden, vocab, xs.data_ptr(), hidden, w.data_ptr(), hidden, tokens.data_ptr(), grad.data_ptr(), 1, loss.data_ptr(), lse.data_ptr(),
                                dx.data_ptr(), hidden, dw.data_ptr(), fp.FT_F32, False, ws.data_ptr(), n, stream()) == 0
    rc, out = run_scores(pool, x, w, tokens, 0, scale)
    # both in fp32: a few roundings of numbers of the size of the sum's logarithm (about 7 and 16)
    assert rc == 0 and float((out["logprob"] + loss).abs().max()) <= 32 * 2.0 ** -24 * 32
    # e is rounded to bf16 (2^-8 of a term), dx once more; x's factor for dw to two bf16 values
    for got, exp, of in ((dx.double() * scale, x64.grad, 2), (dw.double(), w64.grad, 1)):
        assert float((got - exp).norm() / exp.norm()) <= of * 2.0 ** -8
