"""Rotary positions, the root-mean-square norm, the gradients' norm and token log probabilities where their kernels change form or
their neighbours differ: offsets beyond 32 bits, few rows that do not count, several streams, captured beside copies, several pieces.
Tolerances as in the 64-bit tests: U is fp32's unit roundoff, B bf16's."""
import math

import numpy as np
import pytest
import torch

from paper_2606_23087_b200 import binding as fp
from test_gpu_more_operators import (BAD_ID, B, U, bits, check_scores, gen, grad_norm, in_order, new_pool, pool, randn, run_scores,  # noqa: F401
                                     score_inputs, stream, within)

pytestmark = pytest.mark.gpu


# ---- offsets beyond 32 bits -------------------------------------------------------------------------------------

def far_rows(n, dtype, stride):
    """[3, n] rows `stride` elements apart in one buffer, its unused part never touched."""
    buf = torch.empty(2 * stride + n + 64, dtype=dtype, device="cuda")
    return torch.as_strided(buf, (3, n), (stride, 1))


@pytest.mark.parametrize("cols", [200, 201])
def test_rms_norm_and_rotary_of_rows_far_apart(pool, cols):  # noqa: F811
    stride = (1 << 31) + 8 if cols % 8 == 0 else (1 << 31) + 7
    g = gen(cols)
    x, y = far_rows(cols, torch.bfloat16, stride), far_rows(cols, torch.bfloat16, stride)
    near = randn(g, 3, cols).bfloat16()
    x.copy_(near)
    rstd = torch.empty(3, device="cuda")
    assert pool.rms_norm(3, cols, x.data_ptr(), stride, 0, 0, fp.FT_BF16, 0, fp.FT_F32, 1e-6, 0, 0, y.data_ptr(), stride, rstd_ptr=rstd.data_ptr(),
                         stream=stream()) == 0
    out = torch.empty_like(near)
    assert pool.rms_norm(3, cols, near.data_ptr(), cols, 0, 0, fp.FT_BF16, 0, fp.FT_F32, 1e-6, 0, 0, out.data_ptr(), cols, stream=stream()) == 0
    e = near.double() * ((near.double() ** 2).mean(1, keepdim=True) + 1e-6) ** -0.5
    within(y, e, (44 * U + 1.001 * B) * e.abs(), "far rows")
    within(out, e, (44 * U + 1.001 * B) * e.abs(), "rows side by side")
    # backward: dx over dy, in place
    n = pool.rms_norm_grad_workspace(3, cols)
    ws, dx, dw, dw2 = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(near), *torch.empty(2, cols, device="cuda")
    for s, gr, d, ld, w in ((x, y, y, stride, dw), (near, out, dx, cols, dw2)):
        assert pool.rms_norm_grad(3, cols, gr.data_ptr(), ld, s.data_ptr(), ld, 0, 0, fp.FT_BF16, 0, fp.FT_F32, rstd.data_ptr(), d.data_ptr(), ld, w.data_ptr(), False,
                                  ws.data_ptr(), n, stream()) == 0
    # the gradient of a norm's own output: sum(a xhat) / cols is its mean square, and what is left is small beside dy
    r = rstd.double()[:, None]
    a, xhat = out.double(), near.double() * r
    e = r * (a - xhat * (a * xhat).mean(1, keepdim=True))
    mag = r * (a.abs() + xhat.abs() * (a * xhat).abs().mean(1, keepdim=True))
    within(dx, e, 80 * U * mag + 1.01 * B * e.abs() + 1e-30, "dx, rows side by side")
    within(y, e, 80 * U * mag + 2 * B * mag + 1e-30, "dx, far rows")   # (its dy was rounded from other sums, at most 2^-8 of it)
    within(dw, dw2, (2 * B) * (a * xhat).abs().sum(0), "dweight")
    if cols % 8 == 0:
        pos = torch.tensor([[3, 5, 100000]], device="cuda", dtype=torch.int32)
        cfg = fp.rotary_config(1e4 ** (-np.arange(16) / 16), None, 40)
        both = [fp.RotaryTensor(src=x.data_ptr(), dst=x.data_ptr(), src_row=stride, src_head=40, dst_row=stride, dst_head=40, heads=5, dtype=fp.FT_BF16),
                fp.RotaryTensor(src=near.data_ptr(), dst=near.data_ptr(), src_row=cols, src_head=40, dst_row=cols, dst_head=40, heads=5, dtype=fp.FT_BF16)]
        assert pool.rotary(3, pos.data_ptr(), 3, cfg, both, stream()) == 0
        assert torch.equal(bits(x), bits(near))


def test_grad_norm_of_more_than_32_bits_of_elements(pool):  # noqa: F811
    n = (1 << 32) + 77
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[5], g[(1 << 32) - 1], g[1 << 32], g[n - 1] = 1, 2, 4, 10
    assert float(grad_norm(pool, [g])[0]) == 121.0
    assert float(grad_norm(pool, [g[1:], g[:6]])[0]) == 122.0


def test_logprobs_in_pieces_of_4_gib(pool):  # noqa: F811
    """At the best workspace the logits that alternatives keep take several pieces, each beyond 32 bits of bytes."""
    rows, hidden, vocab, top = 3700, 8, 300001, 2
    x, w, tokens = score_inputs(31, rows, hidden, vocab, 0.95)
    rc, out = run_scores(pool, x, w, tokens, top)
    assert rc == 0
    for at in (0, 1500, 3300):
        part = slice(at, at + 300)
        check_scores({k: v[part] for k, v in out.items()}, x[part], w, tokens[part], top, 1.0)
    rc, only = run_scores(pool, x, w, tokens, 0)
    assert rc == 0
    for k in ("logprob", "entropy"):
        within(only[k], out[k], 1e-30, k)


# ---- few rows ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows", [1, 16, 33, 64, 65, 128, 129, 256, 300])
def test_rows_that_do_not_count_reach_nothing(pool, rows):  # noqa: F811
    x, w, tokens = score_inputs(rows, rows, 264, 3001, 1.0)
    x = x.clone()
    clean = run_scores(pool, x, w, tokens, 6)[1]
    for i in range(0, rows, 3):
        x[i] = float("nan") if i % 2 else float("inf")
        tokens[i] = -100
    if rows > 8:
        tokens[4], tokens[7] = 3001, -5
    rc, out = run_scores(pool, x, w, tokens, 6)
    assert rc == 0
    assert pool.status() == ((BAD_ID, 4) if rows > 8 else (0, 0))
    keep = (tokens >= 0) & (tokens < 3001)
    for k in out:
        assert torch.equal(bits(out[k][keep]), bits(clean[k][keep])), k
        assert (out[k][~keep] == (-1 if k == "ids" else 0)).all(), k


@pytest.mark.parametrize("vocab", [1, 31, 32, 33, 128, 129, 4736, 4737, 19000])
@pytest.mark.parametrize("hidden", [8, 1024, 1088, 4104, 4232])
def test_few_rows_at_the_ends_of_tiles_and_parts(pool, vocab, hidden):  # noqa: F811
    """Vocabularies that leave a CTA one segment, or none, and K in one part, a whole one and a little, and several."""
    for rows, top in ((5, 8), (64, 0), (40, 32), (128, 4), (256, 1)):
        x, w, tokens = score_inputs(rows + vocab, rows, hidden, vocab, 0.9, hidden + 8, hidden)
        rc, out = run_scores(pool, x, w, tokens, top)
        assert rc == 0
        check_scores(out, x, w, tokens, top, 1.0)


def test_pieces_of_as_many_rows_as_count_as_few(pool):  # noqa: F811
    """The least workspace for 300 rows holds 256 at a time: a piece of that size is not a call of few rows."""
    x, w, tokens = score_inputs(14, 300, 128, 900, 0.9)
    first = run_scores(pool, x, w, tokens, 3)[1]
    rc, out = run_scores(pool, x, w, tokens, 3, ws_bytes=lambda least, best: least, fill=255)
    assert rc == 0
    for k in out:
        assert torch.equal(bits(out[k]), bits(first[k])), k


@pytest.mark.parametrize("rows", [64, 65, 128, 129, 256, 257, 512, 513])
def test_scores_do_not_depend_on_the_row_count_s_kernel(pool, rows):  # noqa: F811
    """The same rows alone, and among so many others that another kernel takes them: the same alternatives, numbers to their roundings."""
    x, w, tokens = score_inputs(3, 600, 512, 2500, 1.0)
    rc, most = run_scores(pool, x, w, tokens, 5)
    rc2, out = run_scores(pool, x[:rows], w, tokens[:rows], 5)
    assert rc == 0 and rc2 == 0
    assert torch.equal(out["ids"], most["ids"][:rows])
    check_scores(out, x[:rows], w, tokens[:rows], 5, 1.0)


# ---- streams and graphs -----------------------------------------------------------------------------------------

def test_calls_at_once_on_two_streams(pool):  # noqa: F811
    """Two streams, a workspace each, nothing between them: the results of the calls alone."""
    sides = [torch.cuda.Stream() for _ in range(2)]
    work = []
    for i in range(2):
        x, w, tokens = score_inputs(50 + i, 700 - 650 * i, 512, 6000, 0.9)
        n = pool.token_logprobs_workspace(x.shape[0], 512, 6000, 4)[1]
        m = pool.rms_norm_grad_workspace(x.shape[0], 512)
        out = [torch.empty(x.shape[0], device="cuda"), torch.empty(x.shape[0], device="cuda"), torch.empty(x.shape[0], 4, dtype=torch.int32, device="cuda"),
               torch.empty(x.shape[0], 4, device="cuda"), torch.empty(x.shape[0], 512, device="cuda", dtype=torch.bfloat16), torch.empty(512, device="cuda"),
               torch.empty(1, device="cuda"), torch.empty(1, device="cuda")]
        work.append((x, w, tokens, out, torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(m, dtype=torch.uint8, device="cuda"),
                     torch.empty(pool.grad_norm_workspace(), dtype=torch.uint8, device="cuda"), torch.ones(x.shape[0], device="cuda")))

    def issue(i, st):
        x, w, tokens, out, ws, ws2, ws3, ones = work[i]
        rows = x.shape[0]
        p = [t.data_ptr() for t in out]
        assert pool.token_logprobs(rows, 512, 6000, x.data_ptr(), 512, w.data_ptr(), 512, tokens.data_ptr(), 1.0, p[0], p[1], 4, p[2], p[3], ws.data_ptr(), ws.numel(), st) == 0
        assert pool.rms_norm_grad(rows, 512, x.data_ptr(), 512, x.data_ptr(), 512, x.data_ptr(), 512, fp.FT_BF16, 0, fp.FT_F32, ones.data_ptr(), p[4], 512, p[5], False,
                                  ws2.data_ptr(), ws2.numel(), st) == 0
        assert pool.grad_norm([fp.GradTensor(grad=p[4], n=rows * 512, dtype=fp.FT_BF16), fp.GradTensor(grad=p[5], n=512, dtype=fp.FT_F32)], 1.0, 0, 0, p[6], p[7],
                              ws3.data_ptr(), ws3.numel(), st) == 0
    alone = []
    for i in range(2):
        issue(i, stream())
        torch.cuda.synchronize()
        alone.append([t.clone() for t in work[i][3]])
        for t in work[i][3]:
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            issue(i, sides[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        for a, b in zip(alone[i], work[i][3]):
            assert torch.equal(bits(a), bits(b))


@pytest.mark.parametrize("before", ["copy", "memset", "other stream", "nothing"])
def test_each_call_captured_behind_something_else(pool, before):  # noqa: F811
    """A graph in which each call's first kernel follows a copy from the host, a memset, another stream's work, or nothing."""
    rows, cols, vocab = 70, 256, 900
    x0, w, tokens = score_inputs(9, rows, cols, vocab, 0.9)
    host = x0.cpu().pin_memory()
    x, weight = torch.zeros_like(x0), torch.ones(cols, device="cuda")
    side = torch.cuda.Stream()
    pos = torch.arange(rows, device="cuda", dtype=torch.int32)
    cfg = fp.rotary_config(1e4 ** (-np.arange(32) / 32), None, 64)
    y, z, dx = (torch.zeros_like(x0) for _ in range(3))
    f = [torch.zeros(n, device="cuda") for n in (rows, cols, 1, 1, rows, rows)]
    sizes = pool.rms_norm_grad_workspace(rows, cols), pool.grad_norm_workspace(), pool.token_logprobs_workspace(rows, cols, vocab, 0)[1]
    ws = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in sizes]
    scratch = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    X, Y, Z, D = (t.data_ptr() for t in (x, y, z, dx))
    F = [t.data_ptr() for t in f]
    turn = [fp.RotaryTensor(src=X, dst=Y, src_row=cols, src_head=64, dst_row=cols, dst_head=64, heads=4, dtype=fp.FT_BF16)]
    calls = [lambda st: pool.rotary(rows, pos.data_ptr(), rows, cfg, turn, st),
             lambda st: pool.rms_norm(rows, cols, Y, cols, 0, 0, fp.FT_BF16, weight.data_ptr(), fp.FT_F32, 1e-6, 0, 0, Z, cols, rstd_ptr=F[0], stream=st),
             lambda st: pool.rms_norm_grad(rows, cols, Z, cols, Y, cols, X, cols, fp.FT_BF16, weight.data_ptr(), fp.FT_F32, F[0], D, cols, F[1], False, ws[0].data_ptr(),
                                           sizes[0], st),
             lambda st: pool.grad_norm([fp.GradTensor(grad=D, n=rows * cols, dtype=fp.FT_BF16)], 1.0, 0, 0, F[2], F[3], ws[1].data_ptr(), sizes[1], st),
             lambda st: pool.token_logprobs(rows, cols, vocab, Z, cols, w.data_ptr(), cols, tokens.data_ptr(), 1.0, F[4], F[5], 0, 0, 0, ws[2].data_ptr(), sizes[2], st)]

    def between(st):
        if before == "copy":
            x.copy_(host, non_blocking=True)
        elif before == "memset":
            scratch.zero_()
        elif before == "other stream":
            side.wait_stream(st)
            with torch.cuda.stream(side):
                scratch.add_(1)
            st.wait_stream(side)

    main = torch.cuda.Stream()
    x.copy_(x0)
    torch.cuda.synchronize()
    for call in calls:
        assert call(stream()) == 0
    torch.cuda.synchronize()
    expect = [t.clone() for t in (y, z, dx, *f)]
    for t in (y, z, dx, *f):
        t.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=main):
        for call in calls:
            between(main)
            assert call(main.cuda_stream) == 0
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(expect, (y, z, dx, *f)):
        assert torch.equal(bits(a), bits(b))


def test_launches_are_counted():
    p = new_pool()
    x = torch.zeros(4, 64, device="cuda")
    before = p.stats()["gpu_launches"]
    assert p.rms_norm(4, 64, x.data_ptr(), 64, 0, 0, fp.FT_F32, 0, fp.FT_F32, 1e-6, 0, 0, x.data_ptr(), 64, stream=stream()) == 0
    ws = torch.empty(p.grad_norm_workspace(), dtype=torch.uint8, device="cuda")
    assert p.grad_norm([fp.GradTensor(grad=x.data_ptr(), n=256, dtype=fp.FT_F32)], 1.0, 0, 0, x.data_ptr(), 0, ws.data_ptr(), ws.numel(), stream()) == 0
    assert p.stats()["gpu_launches"] == before + 3
    torch.cuda.synchronize()
    p.destroy()


def test_entropy_and_alternatives_without_given_tokens_at_many_temperatures(pool):  # noqa: F811
    x, w, _ = score_inputs(77, 30, 128, 2000, 1.0)
    for scale in (1e-30, 0.01, 1.0, 7.5, 1e4):
        rc, out = run_scores(pool, x, w, None, 3, scale)
        assert rc == 0
        z = x.double() @ w.double().T
        logp = torch.log_softmax(z * float(np.float32(scale)), 1)
        exp = -torch.nan_to_num(logp.exp() * logp).sum(1)
        spread = scale * (z.amax(1) - z.amin(1)).clamp(max=400 / scale)
        # an exponent's product is off by 2^-23 of it, which the terms that still count have below 400
        tol = (64 + 40) * U * (1 + math.log(2000)) + 8 * U * spread + 40 * U * exp
        within(out["entropy"], exp, tol * 4, f"entropy at {scale}")
        assert torch.equal(out["ids"].long(), in_order(z, 3))
