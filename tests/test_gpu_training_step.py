"""The operators of the backbone's last layer together with the pool: whole steps on the tied table (the example), one step's
gradient against a plain 64-bit model, and the token loss's bounded waits."""
import os
import sys

import pytest
import torch

from paper_2606_23087_b200 import binding as fp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
import tied_table_step  # noqa: E402
import workloads  # noqa: E402

pytestmark = pytest.mark.gpu


def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_bring_the_loss_down(bits):
    _gpu()
    losses = tied_table_step.train("tiny", samples=6, hidden=256, steps=6, state_bits=bits)
    assert all(a > b for a, b in zip(losses, losses[1:])), losses


def test_a_step_s_gradients_against_a_plain_model():
    """The gradient of the mean loss for table, gain and shift, by 64-bit autograd over all microbatches.  On the way the
    library rounds six times to bf16 (normalised rows, probabilities, a row's factor times x, dx, the norm's dx, and the norm's
    output in dw); each rounding is at most 2^-8 of what it rounds, so in the norm the results are off by at most 6 x 2^-8 plus
    what is rounded elsewhere, which 8 x 2^-8 covers."""
    _gpu()
    w = workloads.make_workload("tiny", n_samples=12, hidden=64)
    run = tied_table_step.TiedTable(w)
    assert run.n_mb > 1
    table = run.master.double().requires_grad_()
    gain, shift = run.gain.double().requires_grad_(), run.shift.double().requires_grad_()
    tokens = run.plan.arrays()["mb_tokens"]
    mean_loss = 0
    for b in range(run.n_mb):
        run.forward_backward(b)
        ids, labels = run.ids.long(), run.labels.long()
        rows = run.embeds.double()
        text = torch.zeros(run.L, dtype=torch.bool, device="cuda")   # a text position's row is its id's row of the table
        text[: int(tokens[b])] = True
        text &= ids != w.placeholder_id
        rows = torch.where(text[:, None], table[ids], rows)
        assert torch.equal(rows.detach(), run.embeds.double())
        h = torch.nn.functional.layer_norm(rows, (run.H,), gain, shift, 1e-5)
        keep = labels != -100
        losses = torch.nn.functional.cross_entropy(h[keep] @ table.T, labels[keep], reduction="none")
        assert torch.equal(run.loss[~keep], torch.zeros_like(run.loss[~keep]))
        # a logit is off by what rounding h brings, at most 2^-8 of sum |h w|; so is a loss, by twice that
        off = 2 * 2.0 ** -8 * (h[keep].abs() @ table.abs().T).max(1).values
        assert ((run.loss[keep].double() - losses).abs() <= off).all()
        mean_loss = mean_loss + losses.sum() / run.n_labels
    mean_loss.backward()
    for got, exp in ((run.g_table, table.grad), (run.g_gain, gain.grad), (run.g_shift, shift.grad)):
        assert float((got.double() - exp).norm() / exp.norm()) <= 8 * 2.0 ** -8
    assert run.pool.status() == (0, 0)
    run.close()


@pytest.mark.parametrize("rows", [100, 600])
def test_a_token_loss_wait_that_runs_out_reports_timeout_and_leaves_the_context_usable(rows):
    """Under the test hook every load announces 16 bytes more than it brings, so no stage is ever seen complete although all
    arrive: every warp of every pair waits a millisecond, gives up, waits once more for what it has under way, and returns."""
    _gpu()
    p = fp.Pool(fp.PoolConfig(page_bytes=4096, hbm_pages=1, max_text_tokens=1024, hidden=8, max_samples=1, max_spans_per_sample=1,
                              max_pages_per_span=1, max_seq_len=1))
    assert p.rc == 0
    hidden, vocab = 136, 1000
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, hidden, device="cuda", generator=g).bfloat16()
    w = torch.randn(vocab, hidden, device="cuda", generator=g).bfloat16()
    labels = torch.randint(0, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
    ws = torch.zeros(p.token_loss_workspace(rows, hidden, vocab, True)[1], dtype=torch.uint8, device="cuda")

    def call():
        out = [torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros_like(x), torch.zeros(vocab, hidden, device="cuda")]
        loss, lse, dx, dw = (t.data_ptr() for t in out)
        assert p.token_loss_grad(rows, hidden, vocab, x.data_ptr(), hidden, w.data_ptr(), hidden, labels.data_ptr(), 0, 0, loss, lse, dx, hidden,
                                 dw, fp.FT_F32, False, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        return out

    first = call()
    assert p.status() == (0, 0)
    assert p.set_tuning(bulk_timeout_test=1, bulk_wait_limit_us=1000) == 0
    call()
    code, detail = p.status()
    assert code == -13, fp.STATUS.get(code)
    assert detail < torch.cuda.get_device_properties(0).multi_processor_count
    assert p.set_tuning() == 0
    again = call()
    assert p.status() == (0, 0)
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    p.destroy()
