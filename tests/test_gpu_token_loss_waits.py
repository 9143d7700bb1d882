"""The token loss's bounded waits under the shortest limit that a pool can be given: a tile's products are waited for as a whole and
may take longer than that, which is no loss."""
import pytest
import torch

from paper_2606_23087_b200 import binding as fp
from test_gpu_operators import gen, randn, run_loss

pytestmark = pytest.mark.gpu


def test_a_short_limit_does_not_end_a_long_product():
    """dx of 2048 rows x 2048 is 64 tiles of 256 rows that sum over 2048 blocks of the vocabulary: 512 cycles a block, 0.5 ms a tile at
    least, under a limit of 0.1 ms."""
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    rows, hidden, vocab = 2048, 2048, 131072
    p = fp.Pool(fp.PoolConfig(page_bytes=4096, hbm_pages=1, max_text_tokens=1024, hidden=8, max_samples=1, max_spans_per_sample=1,
                              max_pages_per_span=1, max_seq_len=1))
    assert p.rc == 0
    g = gen(1)
    x, w = randn(g, rows, hidden).bfloat16(), (0.02 * randn(g, vocab, hidden)).bfloat16()
    labels = torch.randint(0, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
    out = []
    for limit in (0, 100):
        assert p.set_tuning(bulk_wait_limit_us=limit) == 0
        dw = torch.empty(vocab, hidden, device="cuda", dtype=torch.bfloat16)
        out.append((*run_loss(p, x, w, labels, dw=dw), dw))
        torch.cuda.synchronize()
        assert p.status() == (0, 0)
    assert all(torch.equal(a, b) for a, b in zip(out[0][1:3], out[1][1:3]))
    assert torch.equal(out[0][3].contiguous(), out[1][3].contiguous()) and torch.equal(out[0][4], out[1][4])
    p.destroy()
