"""Token log probabilities of ordinary values, whose sums of products are not exact: how far the numbers are off on average, and that
what a call says about a token is one number.

The tensor cores truncate at every addition of 16 products, all one way, so errors of that kind do not average out.  A model of it on the
CPU (each 16 products added exactly to the sum, then cut to fp32; 64 rows, 2048 columns) gives as mean relative errors of a log probability,
with the given token's logit taken from those sums / from exact ones:
    tokens at random,  K = 1024  1.5e-7 / 1.3e-7;  4096 in parts of 1024  1.3e-7 / 1.3e-7;  4224 in one piece  7.7e-7 / 6.0e-7
    likely tokens,     K = 1024  6.5e-6 / 7.5e-7;  4096 in parts of 1024  6.0e-6 / 6.9e-7;  4224 in one piece  2.8e-5 / 3.4e-6
and of the likeliest alternative 6.4e-7 (1024), 5.8e-7 (parts), 2.8e-6 (one piece) where all logits carry it.  The bounds are about twice
the second numbers, for what fp32 rounds besides."""
import pytest
import torch

from test_gpu_more_operators import bits, gen, pool, randn, run_scores  # noqa: F401

pytestmark = pytest.mark.gpu


def inputs(seed, rows, hidden, vocab, likely):
    """Ordinary values; `likely`: x leans towards its token's row, as a trained model's does."""
    g = gen(seed)
    w = (randn(g, vocab, hidden) * hidden ** -0.5).bfloat16()
    tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
    x = randn(g, rows, hidden)
    if likely:
        x += 8 * w[tokens.long()].float()
    return x.bfloat16(), w, tokens


def truth(x, w, scale=1.0):
    z = x.double() @ w.double().T * scale
    logp = z - torch.logsumexp(z, 1, keepdim=True)
    return logp, -(logp.exp() * logp).sum(1)


def mean_error(got, exp):
    return float(((got.double() - exp).abs() / exp.abs()).mean())


# rows, hidden, vocab, whether a logit's K is summed in parts of 1024
SHAPES = [(24, 1024, 4001, True), (24, 4096, 4001, True), (64, 4096, 4001, True), (300, 4104, 3001, True), (2000, 4104, 20011, False)]


def check_precision(pool, rows, hidden, vocab, parts, likely):  # noqa: F811
    x, w, tokens = inputs(rows + hidden, rows, hidden, vocab, likely)
    logp, entropy = truth(x, w)
    picked = logp.gather(1, tokens.long()[:, None])[:, 0]
    bound = (1.5e-6 if parts else 7e-6) if likely else (3e-7 if parts else 1.2e-6)
    for top in (0, 8):
        rc, out = run_scores(pool, x, w, tokens, top)
        assert rc == 0
        assert mean_error(out["logprob"], picked) <= bound, (top, mean_error(out["logprob"], picked))
        if top:
            best = logp.topk(top, 1).values
            assert mean_error(out["top"][:, 0], best[:, 0]) <= bound, mean_error(out["top"][:, 0], best[:, 0])
            assert mean_error(out["top"], best) <= bound, mean_error(out["top"], best)
            assert mean_error(out["entropy"], entropy) <= bound, mean_error(out["entropy"], entropy)


@pytest.mark.parametrize("likely", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_numbers_of_ordinary_values(pool, shape, likely):  # noqa: F811
    check_precision(pool, *shape, likely)


@pytest.mark.parametrize("likely", [False, True])
@pytest.mark.parametrize("rows,hidden,vocab", [(100, 4096, 4001), (128, 4224, 4001), (129, 4096, 4001), (200, 4096, 4001), (256, 4224, 4001), (256, 12296, 1001), (40, 20488, 1001),
                                               (5, 40008, 501)])
def test_few_rows_are_summed_in_parts(pool, rows, hidden, vocab, likely):  # noqa: F811
    """Up to 256 rows no more than 1024 of K in one piece, however many rows and however long K."""
    check_precision(pool, rows, hidden, vocab, True, likely)


@pytest.mark.parametrize("likely", [False, True])
@pytest.mark.parametrize("rows,hidden,vocab", [(24, 4096, 5000), (200, 1032, 777), (1000, 1032, 20011)])
def test_a_token_s_number_is_one_number(pool, rows, hidden, vocab, likely):  # noqa: F811
    """The same bits in both outputs where the token is listed, the list in the order of its numbers, and no token left out of it whose
    number is larger than the last one's."""
    x, w, tokens = inputs(rows + vocab, rows, hidden, vocab, likely)
    w[vocab // 2:vocab // 2 * 2] = w[:vocab // 2].clone()   # twins: equal logits, by ascending id
    rc, out = run_scores(pool, x, w, tokens, 8)
    assert rc == 0
    hit = out["ids"] == tokens[:, None]
    assert hit.any() or not likely
    assert torch.equal(bits(out["top"][hit]), bits(out["logprob"][:, None].expand(-1, 8)[hit]))
    assert (out["top"][:, 1:] <= out["top"][:, :-1]).all() and (out["top"] <= 1e-6).all()
    assert (out["logprob"][~hit.any(1)] <= out["top"][~hit.any(1), -1]).all()
    ids = out["ids"].long()
    assert all(len(set(r)) == 8 for r in ids.tolist())
    twins = (ids[:, :-1] % (vocab // 2) == ids[:, 1:] % (vocab // 2)) & (ids.max(1, keepdim=True).values < vocab // 2 * 2)
    assert twins.any()
    assert torch.equal(bits(out["top"][:, :-1][twins]), bits(out["top"][:, 1:][twins])) and (ids[:, :-1][twins] < ids[:, 1:][twins]).all()


@pytest.mark.parametrize("rows,hidden,vocab", [(24, 1024, 3000), (2000, 1032, 20011)])
def test_certain_tokens(pool, rows, hidden, vocab):  # noqa: F811
    """A token whose probability is all but one: its log probability is what the others leave, not a difference of two large numbers."""
    x, w, tokens = inputs(rows, rows, hidden, vocab, False)
    x = (x.float() * 0.5 + 24 * w[tokens.long()].float()).bfloat16()   # logits about 24 against 0.5: log probabilities about -1e-7 to -1e-6
    logp, _ = truth(x, w)
    picked = logp.gather(1, tokens.long()[:, None])[:, 0]
    for top in (0, 4):
        rc, out = run_scores(pool, x, w, tokens, top)
        assert rc == 0
        # the token's logit is summed in 32 lanes of hidden / 32 products, 37 roundings of 24 at the most, the others' in 65 of 2: 5e-5 + 8e-6
        assert mean_error(out["logprob"], picked) <= 6e-5, (top, mean_error(out["logprob"], picked))
    rc, out = run_scores(pool, x, w, None, 1)   # as an alternative: additions to one, in a segment, over segments and in the join
    assert rc == 0 and float((out["top"][:, 0].double() - picked).abs().max()) <= (64 + vocab / 32 / 32 + 16) * 2.0 ** -24
