"""Token log probabilities with alternatives of more than 256 rows, whose results come from a kernel behind the join: captured and replayed on other
inputs, in several pieces, with W and x beyond 32 bits of elements, and rows that do not count among them."""
import pytest
import torch

from test_gpu_logprobs_precision import mean_error
from test_gpu_more_operators import bits, check_scores, pool, run_scores, score_inputs  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,top", [(300, 8), (1300, 1), (2600, 32), (200, 8)])
def test_captured_and_replayed_on_other_inputs(pool, rows, top):  # noqa: F811
    hidden, vocab = 136, 3001
    sets = [score_inputs(rows + i, rows, hidden, vocab, 0.8) for i in range(3)]
    alone = [run_scores(pool, *s, top)[1] for s in sets]
    x, w, tokens = [t.clone() for t in sets[0]]
    out = {k: torch.empty_like(t) for k, t in alone[0].items()}
    n = pool.token_logprobs_workspace(rows, hidden, vocab, top)[1]
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        assert pool.token_logprobs(rows, hidden, vocab, x.data_ptr(), hidden, w.data_ptr(), hidden, tokens.data_ptr(), 1.0, out["logprob"].data_ptr(), out["entropy"].data_ptr(),
                                   top, out["ids"].data_ptr(), out["top"].data_ptr(), ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream) == 0
    for i in (0, 1, 2, 0):
        for t, s in zip((x, w, tokens), sets[i]):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(bits(out[k]), bits(alone[i][k])), (i, k)
    assert pool.status() == (0, 0)


@pytest.mark.parametrize("top", [1, 5, 31])
def test_pieces_with_rows_that_do_not_count(pool, top):  # noqa: F811
    """The least workspace: pieces of 256 rows, some of them with few rows that count, one with none."""
    x, w, tokens = score_inputs(77 + top, 1500, 200, 2003, 0.7)
    x = x.clone()
    tokens[256:512] = -100
    tokens[520:767] = -100
    x[tokens < 0] = float("nan")
    rc, out = run_scores(pool, x, w, tokens, top, ws_bytes=lambda least, best: least, fill=255)
    assert rc == 0
    check_scores(out, x, w, tokens, top, 1.0)
    x[tokens < 0] = 0   # every row counts
    rc, out = run_scores(pool, x, w, None, top, ws_bytes=lambda least, best: least, fill=255)
    assert rc == 0
    check_scores(out, x, w, None, top, 1.0)
    assert pool.status() == (0, 0)


@pytest.mark.parametrize("rows", [5, 300])
def test_rows_of_w_and_x_beyond_32_bits(pool, rows):  # noqa: F811
    hidden, vocab, top = 4096, 540000, 8   # 2.2e9 elements of W; x's rows lie as far apart
    g = torch.Generator(device="cuda").manual_seed(rows)
    w = torch.empty(vocab, hidden, device="cuda", dtype=torch.bfloat16).normal_(0, hidden ** -0.5, generator=g)
    stride = ((1 << 31) // (rows - 1) // 8 + 1) * 8 + 8
    near = torch.randn(rows, hidden, device="cuda", generator=g).bfloat16()
    buf = torch.empty((rows - 1) * stride + hidden, device="cuda", dtype=torch.bfloat16)
    x = torch.as_strided(buf, (rows, hidden), (stride, 1))
    x.copy_(near)
    tokens = torch.randint(vocab - 1000, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
    rc, out = run_scores(pool, x, w, tokens, top)
    assert rc == 0
    z = torch.cat([near.double() @ w[i:i + 60000].double().T for i in range(0, vocab, 60000)], 1)
    lse = torch.logsumexp(z, 1)
    assert mean_error(out["logprob"], z.gather(1, tokens.long()[:, None])[:, 0] - lse) <= 1.2e-6
    best = z.topk(top, 1)
    assert mean_error(out["top"], best.values - lse[:, None]) <= 1.2e-6
    assert (out["ids"][:, 0].long() == best.indices[:, 0]).float().mean() >= 0.9   # (ties to fp32 aside)
    own = z.gather(1, out["ids"].long()) - lse[:, None]   # each listed id's own number
    assert mean_error(out["top"], own) <= 1.2e-6
