"""Rotary positions, the root-mean-square norm, the gradients' norm and token log probabilities together with the pool, as a step on the
tied table uses them (the example), against plain 64-bit models."""
import os
import sys

import numpy as np
import pytest
import torch

from paper_2606_23087_b200 import binding as fp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
import tied_table_step  # noqa: E402
import workloads  # noqa: E402

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8


def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_with_the_root_mean_square_norm_and_clipping_run(bits):
    _gpu()
    losses = tied_table_step.train("tiny", samples=6, hidden=256, steps=3, state_bits=bits, norm="rms", max_norm=0.5)
    assert len(losses) == 3 and np.isfinite(losses).all()


def test_a_step_s_gradients_norm_and_clipped_update_against_a_plain_model():
    """The gradient of the mean loss for table and gain by 64-bit autograd over all microbatches, its norm, and the step that AdamW takes
    with the gradients clipped.  On the way the library rounds six times to bf16 (normalised rows, probabilities, a row's factor times x,
    dx, the norm's dx, and the norm's output in dw); each rounding is at most 2^-8 of what it rounds, so in the norm the results are off by
    at most 6 x 2^-8 plus what is rounded elsewhere, which 8 x 2^-8 covers."""
    _gpu()
    w = workloads.make_workload("tiny", n_samples=12, hidden=64)
    run = tied_table_step.TiedTable(w, norm="rms", max_norm=1e-3)
    assert run.n_mb > 1
    before = run.master.clone()
    table = run.master.double().requires_grad_()
    gain = run.gain.double().requires_grad_()
    tokens = run.plan.arrays()["mb_tokens"]
    mean_loss = 0
    for b in range(run.n_mb):
        run._gather(b)
        ids, labels = run.ids.long(), run.labels.long()
        text = torch.zeros(run.L, dtype=torch.bool, device="cuda")   # a text position's row is its id's row of the table
        text[: int(tokens[b])] = True
        text &= ids != w.placeholder_id
        rows = torch.where(text[:, None], table[ids], run.embeds.double())
        h = rows * ((rows * rows).mean(1, keepdim=True) + 1e-5) ** -0.5 * gain
        keep = labels != -100
        mean_loss = mean_loss + torch.nn.functional.cross_entropy(h[keep] @ table.T, labels[keep], reduction="sum") / run.n_labels
    mean_loss.backward()
    loss = float(run.step())
    mean_loss = float(mean_loss.detach())
    assert abs(loss - mean_loss) <= 2 * B * mean_loss   # rounding the normalised rows moves a logit by 2^-8 of itself
    for got, exp in ((run.g_table, table.grad), (run.g_gain, gain.grad)):
        assert float((got.double() - exp).norm() / exp.norm()) <= 8 * B
    # the norm and the factor are those of the gradients as the library has them, to fp32's roundings
    norm = float(torch.cat([run.g_table.double().flatten(), run.g_gain.double()]).norm())
    assert norm > 1e-3
    assert abs(float(run.grad_norm) - norm) <= 12 * U * norm
    assert abs(float(run.clip) - 1e-3 / norm) <= 13 * U * 1e-3 / norm
    # AdamW's first step from zero states: g / (|g| + eps) with the clipped g, so where |g| is well above eps a step of lr
    g = run.g_table.double() * run.clip.double()
    exp = before.double() * (1 - 2e-3 * 0.1) - 2e-3 * g / (g.abs() + 1e-8)
    assert float((run.master.double() - exp).abs().max()) <= 2e-3 * 64 * U + 4 * U * float(exp.abs().max())
    assert run.pool.status() == (0, 0)
    run.close()


def test_scores_of_a_microbatch_against_a_plain_model():
    _gpu()
    w = workloads.make_workload("tiny", n_samples=8, hidden=128)
    run = tied_table_step.TiedTable(w, norm="rms")
    for b in range(run.n_mb):
        logprob, entropy, ids, top = run.score(b, top=5)
        keep = run.labels >= 0
        assert keep.any() and not keep.all()
        z = run.hidden[keep].double() @ run.table.double().T
        logp = torch.log_softmax(z, 1)
        # a logit of 128 products is off by at most 2 U (128 + 8) of the sum of their magnitudes, a row's lse by that and the exponentials'
        off = 2 * (2 * U * 136 * (run.hidden[keep].double().abs() @ run.table.double().abs().T).amax(1) + (80 + 0.02 * w.vocab) * U * 17)
        labels = run.labels[keep].long()
        assert ((logprob[keep].double() - logp.gather(1, labels[:, None])[:, 0]).abs() <= off).all()
        assert ((entropy[keep].double() + (logp.exp() * logp).sum(1)).abs() <= 2 * off * (1 + np.log(w.vocab))).all()
        best = logp.topk(5, 1).values
        assert ((top[keep].double() - best).abs() <= off[:, None]).all()
        assert ((logp.gather(1, ids[keep].long()) - best).abs() <= 2 * off[:, None]).all()
        assert (logprob[~keep] == 0).all() and (ids[~keep] == -1).all()
        # the loss of the same rows
        run.forward_backward(b)
        assert ((run.loss[keep].double() + logprob[keep].double()).abs() <= 2 * off).all()
    assert run.pool.status() == (0, 0)
    run.close()


def test_rotary_takes_the_positions_that_padded_assembly_writes():
    """Queries and keys turned by out_pos3 as the pool writes it, grids and all: scores between two rows depend on the differences of their
    positions alone, so shifting every position changes none of them."""
    _gpu()
    w = workloads.make_workload("tiny", n_samples=6, hidden=64)
    run = tied_table_step.TiedTable(w)
    slots, spans, grids = [], [], []
    for s in range(6):
        for j in range(int(w.n_spans[s])):
            grid = workloads.span_grid(w, s, j)
            if grid is not None:
                slots.append(s)
                spans.append(j)
                grids.append(grid)
    assert slots
    assert run.pool.set_span_grids(slots, spans, grids, run._stream()) == 0
    run._gather(0)
    pos = run.pos3
    assert not torch.equal(pos[0], pos[2])   # the axes differ somewhere
    L, heads, dim, pairs = run.L, 2, 32, 12
    freqs, axes = 1e4 ** (-np.arange(pairs) / pairs), np.repeat([0, 1, 2], [4, 4, 4])
    g = torch.Generator(device="cuda").manual_seed(1)
    qk = torch.randn(2, L, heads, dim, device="cuda", generator=g)

    def turn(p):
        out = torch.empty_like(qk)
        tensors = [fp.RotaryTensor(src=qk[i].data_ptr(), dst=out[i].data_ptr(), src_row=heads * dim, src_head=dim, dst_row=heads * dim,
                                   dst_head=dim, heads=heads, dtype=fp.FT_F32) for i in range(2)]
        assert run.pool.rotary(L, p.data_ptr(), L, fp.rotary_config(freqs, axes, dim), tensors, run._stream()) == 0
        return out.double()
    angle = pos.double()[torch.as_tensor(axes, device="cuda")].T * torch.as_tensor(freqs, device="cuda")
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = qk[..., :pairs].double(), qk[..., pairs:2 * pairs].double()
    out = turn(pos)
    exp = torch.cat([a * c - b * s, a * s + b * c, qk[..., 2 * pairs:].double()], -1)
    assert ((out - exp).abs() <= 12 * U * 8).all()
    n = min(L, 300)
    near = torch.einsum("ihd,jhd->hij", out[0, :n], out[1, :n])
    far = turn(pos + torch.tensor([[1000], [500000], [7]], device="cuda", dtype=torch.int32))
    assert (near - torch.einsum("ihd,jhd->hij", far[0, :n], far[1, :n])).abs().max() <= dim * 2 * 24 * U * 25
    assert run.pool.status() == (0, 0)
    run.close()
