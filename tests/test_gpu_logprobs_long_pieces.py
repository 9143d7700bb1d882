"""Token log probabilities of pieces so long that their rows are dealt out to CTAs in other numbers: whole and ragged ends, rows that do not count."""
import pytest
import torch

from test_gpu_more_operators import bits, check_scores, pool, run_scores, score_inputs  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("valid", [1.0, 0.4])
@pytest.mark.parametrize("rows", [16383, 16384, 16391, 65537])
def test_rows_of_long_pieces(pool, rows, valid):  # noqa: F811
    x, w, tokens = score_inputs(rows, rows, 72, 301, valid)
    x = x.clone()
    x[tokens < 0] = float("nan")
    rc, out = run_scores(pool, x, w, tokens, 2)
    assert rc == 0
    check_scores(out, x, w, tokens, 2, 1.0)
    for r0 in (0, rows - 300):   # the same rows by themselves
        rc, part = run_scores(pool, x[r0:r0 + 300], w, tokens[r0:r0 + 300], 2)
        assert rc == 0 and torch.equal(part["ids"], out["ids"][r0:r0 + 300])
