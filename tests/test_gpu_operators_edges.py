"""The operators of the last layer and of the optimizer where their kernels change form: sums in parts of K, several row tiles of
which some need another reference, second tiles of a CTA pair, pieces, rows enough to go round a ring.
Helpers and bounds are test_gpu_operators'."""
import pytest
import torch

from test_gpu_norm_wide_access import forward
from test_gpu_operators import (B, loss_formula, loss_inputs, pool, run_loss, same_bits,  # noqa: F401
                                test_layer_norm_grad_against_64_bits as norm_grad_against_64_bits, within)

pytestmark = pytest.mark.gpu


# ---- layer norm -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(1, 8), (5, 64), (33, 1000), (300, 1024), (20000, 256), (6000, 3584), (149, 4096), (3000, 8192)])
def test_layer_norm_in_wide_accesses(pool, shape, dtype):  # noqa: F811
    forward(pool, *shape, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(20000, 256), (6000, 3584), (2000, 8192)])
def test_layer_norm_grad_round_its_ring(pool, shape, dtype):  # noqa: F811
    norm_grad_against_64_bits(pool, shape, dtype)


# ---- token loss -------------------------------------------------------------------------------------------------

def against_64_bits(pool, x, w, labels, grad=None, e=None):  # noqa: F811
    rows, hidden = x.shape
    vocab = w.shape[0]
    e = e or loss_formula(x, w, labels, torch.ones(1, device="cuda") if grad is None else grad)
    rc, loss, lse, _ = run_loss(pool, x, w, labels, fill=255)
    assert rc == 0
    within(loss, e["loss"], e["t_loss"], "loss")
    within(lse, e["lse"], e["t_lse"], "lse")
    for dtype in (torch.float32, torch.bfloat16):
        dw = torch.full((vocab, hidden), float("nan"), device="cuda", dtype=dtype)
        rc, loss2, lse2, dx = run_loss(pool, x, w, labels, grad, 0, dw, fill=255)
        assert rc == 0 and torch.equal(loss2, loss) and torch.equal(lse2, lse)
        within(dx, e["dx"], e["t_dx"] * 1.01 + 1.01 * B * e["dx"].abs() + 1e-30, "dx")
        within(dw, e["dw"], e["t_dw"] * 1.01 + (1.01 * B * e["dw"].abs() if dtype == torch.bfloat16 else 0) + 1e-30, "dw")
        again = torch.full_like(dw, float("nan"))
        rc, loss3, _, dx3 = run_loss(pool, x, w, labels, grad, 0, again)
        assert rc == 0 and torch.equal(loss3, loss) and same_bits(dx3, dx) and same_bits(again, dw)
    return loss


@pytest.mark.parametrize("shape", [
    (200, 1536, 1000, 1.0), (120, 3592, 700, 0.8), (5, 4352, 3000, 1.0), (300, 4352, 600, 0.9), (700, 4232, 520, 0.7),  # parts of K
    (4500, 64, 300, 0.6),       # picked 32 rows a CTA; several row tiles of dx from one slice of a short vocabulary
    (5000, 2056, 3000, 1.0),    # more tiles than pairs in the logits (in three bands of rows) and in dx
    (3000, 1032, 12000, 0.9),   # more 512-row tiles than pairs in dw
    (70000, 8, 64, 0.9),        # two pieces
], ids=str)
def test_token_loss_where_products_change_form(pool, shape):  # noqa: F811
    rows, hidden, vocab, valid = shape
    x, w, labels = loss_inputs(rows * 7 + vocab, rows, hidden, vocab, valid, hidden + 8, hidden + 16)
    against_64_bits(pool, x, w, labels)


@pytest.mark.parametrize("rows, hidden", [(900, 64), (900, 4352), (256, 1536), (1300, 520)])
def test_some_row_tiles_take_another_reference(pool, rows, hidden):  # noqa: F811
    """Rows of every second tile of 256 have a loss above 41, the others none; in the last tile it is the last row alone."""
    vocab = 1111
    x, w, labels = loss_inputs(rows + hidden, rows, hidden, vocab, 1.0)
    far = [r for r in (256, 300, 511, 768, 769, 800) if r < rows - 1] + [rows - 1]
    near = torch.ones(rows, dtype=torch.bool, device="cuda")
    near[far] = False
    other = (labels.long() + vocab // 2) % vocab
    x = torch.where(near[:, None], x, (90 * w[other].float()).bfloat16())
    e = loss_formula(x, w, labels, torch.full((1,), 0.25, device="cuda"))
    assert e["loss"][~near].min() > 45 and e["loss"][near].max() < 38
    against_64_bits(pool, x, w, labels, torch.full((1,), 0.25, device="cuda"), e)
