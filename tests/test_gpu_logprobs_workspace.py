"""Workspaces of token log probabilities: one that serves some rows serves fewer, as a scoring loop's last batch needs it."""
import pytest
import torch

from test_gpu_logprobs_precision import inputs, mean_error, truth
from test_gpu_more_operators import CAPACITY, check_scores, pool, run_scores, score_inputs  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hidden,vocab,top", [(8, 1, 0), (8, 33, 1), (1024, 131072, 0), (1024, 131072, 8), (1024, 32768, 0), (3584, 152064, 8), (40000, 300, 0), (64, 5003, 20), (136, 777, 32)])
def test_fewer_rows_need_no_more(pool, hidden, vocab, top):  # noqa: F811
    last = (0, 0)
    for rows in (0, 1, 2, 31, 32, 33, 64, 65, 128, 129, 200, 255, 256, 257, 300, 512, 1000, 4096, 16384, 70000):
        least, best = pool.token_logprobs_workspace(rows, hidden, vocab, top)
        assert last[0] <= least <= best, rows   # so any size that serves these rows serves the fewer ones
        last = (least, best)


@pytest.mark.parametrize("hidden,vocab,top", [(64, 5003, 0), (64, 5003, 8), (1032, 9001, 0)])
@pytest.mark.parametrize("many", [257, 512, 16384])
def test_the_last_batch_of_a_loop(pool, many, hidden, vocab, top):  # noqa: F811
    """Fewer rows in a workspace made for `many`, the best and the least."""
    x, w, tokens = score_inputs(many + vocab, 256, hidden, vocab, 0.9)
    for which in (0, 1):
        n = pool.token_logprobs_workspace(many, hidden, vocab, top)[which]
        for rows in (256, 200, 33, 1):
            rc, out = run_scores(pool, x[:rows], w, tokens[:rows], top, ws_bytes=lambda *_: n, fill=255)
            assert rc == 0, (which, rows)
            check_scores(out, x[:rows], w, tokens[:rows], top, 1.0)
    least = pool.token_logprobs_workspace(200, hidden, vocab, top)[0]
    assert run_scores(pool, x[:200], w, tokens[:200], top, ws_bytes=lambda *_: least)[0] == 0
    assert run_scores(pool, x[:200], w, tokens[:200], top, ws_bytes=lambda *_: least - 1)[0] == CAPACITY


@pytest.mark.parametrize("rows,top", [(2000, 0), (2000, 8), (256, 8)])
def test_the_size_of_the_workspace_changes_roundings_alone(pool, rows, top):  # noqa: F811
    """Ordinary values: by tiles of 512 rows, of 256 and as few rows, as the workspace has room; the bound is that of K = 4104 in one piece."""
    x, w, tokens = inputs(rows, rows, 4104, 20011, False)
    logp, _ = truth(x, w)
    picked = logp.gather(1, tokens.long()[:, None])[:, 0]
    for n in (lambda least, best: least, lambda least, best: (least + best) // 2, lambda least, best: best):
        rc, out = run_scores(pool, x, w, tokens, top, ws_bytes=n)
        assert rc == 0 and mean_error(out["logprob"], picked) <= 1.2e-6
        if top:
            assert mean_error(out["top"], logp.topk(top, 1).values) <= 1.2e-6
