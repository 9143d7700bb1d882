"""logit_scale over all that fp32 holds: near its largest value the likeliest token alone counts, near zero all of them count alike."""
import pytest
import torch

from test_gpu_logprobs_precision import inputs
from test_gpu_more_operators import U, in_order, pool, run_scores, score_inputs, within  # noqa: F401

pytestmark = pytest.mark.gpu
LARGEST = float(torch.finfo(torch.float32).max)


@pytest.mark.parametrize("rows", [5, 300])
@pytest.mark.parametrize("scale", [LARGEST, 2.4e38, 2.3e38, 1e30, 1e6, 1e-6, 1e-30, 1e-45])
def test_scores_at_extreme_scales(pool, rows, scale):  # noqa: F811
    """The logits are exact: a difference of two is rounded once, its product with the scale once, as is the sum's logarithm."""
    x, w, tokens = score_inputs(rows, rows, 64, 700, 1.0)
    scale = float(torch.tensor(scale, dtype=torch.float32))
    z = x.double() @ w.double().T * scale
    logp = z - torch.logsumexp(z, 1, keepdim=True)
    p = logp.exp()
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
    rc, out = run_scores(pool, x, w, tokens, 4, scale)
    assert rc == 0
    best = in_order(x.double() @ w.double().T, 4)
    assert torch.equal(out["ids"].long(), best)
    for got, exp in ((out["logprob"], logp.gather(1, tokens.long()[:, None])[:, 0]), (out["top"], logp.gather(1, best))):
        over = exp < -LARGEST
        assert (got[over] < -1e38).all()
        # differences of scaled logits in 64 bits are off by 2^-53 of those
        within(got[~over], exp[~over], (64 + 0.02 * 700 + 8 * 16) * U + 8 * U * exp[~over].abs() + 2.0 ** -50 * float(z.abs().max()), "numbers")
    # a term's exponent is off by 3 U of it, and what is left of it times its probability is at most 1 / e; then the sums
    within(out["entropy"], entropy, (64 + 0.02 * 700 + 40 * 16) * U * (1 + entropy) + 2.0 ** -50 * float(z.abs().max()) * (p * (1 - p)).sum(1), "entropy")


@pytest.mark.parametrize("negative", [False, True])
@pytest.mark.parametrize("rows", [5, 300])
@pytest.mark.parametrize("top", [0, 1, 8, 32])
@pytest.mark.parametrize("scale", [1e2, 1e4, 1e5, 1e6, 1e7, 1e9, 1e20, LARGEST])
def test_ordinary_values_at_large_scales(pool, rows, top, scale, negative):  # noqa: F811
    """Scales at which a logit's rounding is worth powers of e: numbers all the same, none above zero, off by what a logit's sum may be off."""
    hidden, vocab = 1032, 1501
    x, w, tokens = inputs(rows, rows, hidden, vocab, True)
    tokens[::2] = (tokens[::2] + 1) % vocab
    if negative:   # cut towards zero, every logit is larger than it should be
        x, w = -x.abs(), w.abs()
    rc, out = run_scores(pool, x, w, tokens, top, scale)
    assert rc == 0
    z = x.double() @ w.double().T
    logp = z * scale - torch.logsumexp(z * scale, 1, keepdim=True)
    bound = 4 * scale * 2 * U * (hidden + 8) * (x.double().abs() @ w.double().abs().T).amax(1) + 1e-4
    picked = logp.gather(1, tokens.long()[:, None])[:, 0]
    real = picked > -LARGEST / 2
    within(out["logprob"][real], picked[real], (bound + 8 * U * picked.abs())[real], "logprob")
    assert not out["logprob"].isnan().any() and (out["logprob"] <= 1e-6).all() and not out["entropy"].isnan().any() and (out["entropy"] >= -1e-5).all()
    if top:
        assert not out["top"].isnan().any() and (out["top"][:, 1:] <= out["top"][:, :-1]).all()
        assert (out["top"].double().exp().sum(1) <= 1 + 1e-5).all()
        first = z.gather(1, out["ids"][:, :1].long())[:, 0]
        assert ((z.amax(1) - first) * scale <= bound).all()
