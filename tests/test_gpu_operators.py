"""The operators of the backbone's last layer and of its optimizer on the GPU, against plain 64-bit implementations of
their formulas.  Every tolerance is an error bound worked out from the formula: U is fp32's unit roundoff, B bf16's; a sum
of n fp32 terms in any order is off by at most n U times the sum of the terms' magnitudes (2 U for the tensor cores, whose
additions may truncate)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2606_23087_b200 import binding as fp

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
INVALID, BAD_ID, CAPACITY = -1, -9, -11


@pytest.fixture(scope="module")
def pool():
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    p = fp.Pool(fp.PoolConfig(page_bytes=4096, hbm_pages=1, max_text_tokens=1024, hidden=8, max_samples=1, max_spans_per_sample=1,
                              max_pages_per_span=1, max_seq_len=1))
    assert p.rc == 0
    yield p
    torch.cuda.synchronize()
    assert p.status() == (0, 0)
    p.destroy()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def stream():
    return torch.cuda.current_stream().cuda_stream


def strided(t, ld, shift=0):
    """A copy of the matrix with row stride ld, `shift` elements into its buffer, the rest NaN."""
    rows, cols = t.shape
    buf = torch.full((rows * ld + shift + 64,), float("nan"), dtype=t.dtype, device="cuda")
    view = torch.as_strided(buf, (rows, cols), (ld, 1), shift)
    view.copy_(t)
    return view


def same_bits(a, b):
    return torch.equal(a.flatten().clone().view(torch.uint8), b.flatten().clone().view(torch.uint8))


def within(got, exp, bound, what):
    got, exp = got.double(), exp.double()
    bad = ~((got - exp).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float(((got - exp).abs() / bound).max()):.3g} times it"


# ---- layer norm -------------------------------------------------------------------------------------------------

EPS = 1e-5
SHAPES = [(1, 1), (3, 1), (1, 8), (5, 31), (33, 64), (7, 129), (300, 1000), (257, 1023), (64, 1024), (1, 3584), (150, 3584), (40, 4096),
          (9, 8192), (12, 8191), (5, 8200), (3, 20001)]


def code(t):
    return fp.FT_BF16 if t == torch.bfloat16 else fp.FT_F32


def norm_bounds(x, w, b, mean, rstd):
    """|y - y'| before the last rounding: 64 roundings in a row's sums, a few in the products"""
    near = 64 * U * x.abs().mean(1, keepdim=True)
    xhat = ((x - mean) * rstd).abs()
    return (w.abs() * (near * rstd + xhat * (near * rstd) ** 2 + xhat * 80 * U)) + 4 * U * (b.abs() + (w * xhat).abs())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES)
def test_layer_norm_against_64_bits(pool, shape, dtype):
    rows, cols = shape
    g = gen(rows * 10007 + cols)
    x = (randn(g, rows, cols) * torch.exp(randn(g, rows, 1)) + randn(g, rows, 1)).to(dtype)
    w, b = 1 + 0.1 * randn(g, cols), 0.1 * randn(g, cols)
    ld = cols + 3 if cols % 2 else cols
    xs, y = strided(x, ld), strided(torch.zeros_like(x), ld + 5)
    mean, rstd = torch.empty(2, rows, device="cuda")
    assert pool.layer_norm(rows, cols, xs.data_ptr(), ld, code(dtype), w.data_ptr(), b.data_ptr(), fp.FT_F32, EPS, y.data_ptr(), ld + 5,
                           mean.data_ptr(), rstd.data_ptr(), stream()) == 0
    x6, w6, b6 = x.double(), w.double(), b.double()
    m6 = x6.mean(1, keepdim=True)
    r6 = (((x6 - m6) ** 2).mean(1, keepdim=True) + EPS) ** -0.5
    e6 = (x6 - m6) * r6 * w6 + b6
    within(mean[:, None], m6, 64 * U * x6.abs().mean(1, keepdim=True) + 1e-30, "mean")
    near = 64 * U * x6.abs().mean(1, keepdim=True) * r6
    within(rstd[:, None], r6, r6 * (80 * U + near + near ** 2), "rstd")
    bound = norm_bounds(x6, w6, b6, m6, r6)
    within(y, e6, bound + (B * (e6.abs() + bound) if dtype == torch.bfloat16 else 2 * U * e6.abs()) + 1e-30, "y")
    # a row's neighbours in memory stay as they were
    gap = torch.as_strided(y, (rows, 5), (ld + 5, 1), y.storage_offset() + cols)
    assert gap.isnan().all()


@pytest.mark.parametrize("cols", [1, 40, 1023, 3584, 9000])
def test_layer_norm_keeps_bad_rows_to_themselves_and_works_in_place(pool, cols):
    g = gen(cols)
    x = randn(g, 6, cols).bfloat16()
    x[1, cols // 2] = float("nan")
    x[3, 0] = float("inf")
    x[4] = 2.5  # a constant row: y is the bias
    w, b = randn(g, cols).bfloat16(), randn(g, cols).bfloat16()
    clean, y = x.clone(), torch.empty_like(x)
    args = (w.data_ptr(), b.data_ptr(), fp.FT_BF16, EPS)
    assert pool.layer_norm(6, cols, clean.data_ptr(), cols, fp.FT_BF16, *args, y.data_ptr(), cols, 0, 0, stream()) == 0
    assert pool.layer_norm(6, cols, clean.data_ptr(), cols, fp.FT_BF16, *args, clean.data_ptr(), cols, 0, 0, stream()) == 0
    assert torch.equal(clean.view(torch.int16), y.view(torch.int16))
    assert y[[1, 3]].isnan().all() and y[[0, 2, 4, 5]].isfinite().all()
    assert torch.equal(y[4], b)
    plain = torch.empty_like(x)  # neither weight nor bias
    assert pool.layer_norm(6, cols, x.data_ptr(), cols, fp.FT_BF16, 0, 0, fp.FT_F32, EPS, plain.data_ptr(), cols, 0, 0, stream()) == 0
    x6 = x[0].double()
    within(plain[0], (x6 - x6.mean()) / (x6.var(unbiased=False) + EPS).sqrt(), 2 * B * 8 + 1e-6, "no weight")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES + [(5000, 136), (2049, 77)])
def test_layer_norm_grad_against_64_bits(pool, shape, dtype):
    rows, cols = shape
    g = gen(rows * 31 + cols)
    x = (randn(g, rows, cols) + 0.5).to(dtype)
    dy, w = randn(g, rows, cols).to(dtype), (1 + 0.1 * randn(g, cols)).to(torch.bfloat16)
    x6, dy6, w6 = x.double(), dy.double(), w.double()
    mean = x6.mean(1).float()
    rstd = (x6.var(1, unbiased=False) + EPS).rsqrt().float()
    ld = cols + 3 if cols % 2 else cols
    xs, gs, dx = strided(x, ld, 1 if cols % 2 else 0), strided(dy, ld + 8), strided(torch.zeros_like(x), ld)
    dw, db = torch.full((2, cols), float("nan"), device="cuda")
    n = pool.layer_norm_grad_workspace(rows, cols)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")

    def call(out, dw, db, add):
        return pool.layer_norm_grad(rows, cols, gs.data_ptr(), ld + 8, xs.data_ptr(), ld, code(dtype), w.data_ptr(), fp.FT_BF16, mean.data_ptr(),
                                    rstd.data_ptr(), out.data_ptr(), ld, dw.data_ptr(), db.data_ptr(), add, ws.data_ptr(), n, stream())

    assert call(dx, dw, db, False) == 0
    r6 = rstd.double()[:, None]
    xhat, a = (x6 - mean.double()[:, None]) * r6, dy6 * w6
    e6 = r6 * (a - a.mean(1, keepdim=True) - xhat * (a * xhat).mean(1, keepdim=True))
    mag = r6 * (a.abs() + a.abs().mean(1, keepdim=True) + xhat.abs() * (a * xhat).abs().mean(1, keepdim=True))
    within(dx, e6, 80 * U * mag + (B * 1.01 * e6.abs() if dtype == torch.bfloat16 else 0) + 1e-30, "dx")
    within(dw, (dy6 * xhat).sum(0), (rows + 16) * U * (dy6 * xhat).abs().sum(0) + 1e-30, "dweight")
    within(db, dy6.sum(0), (rows + 16) * U * dy6.abs().sum(0) + 1e-30, "dbias")
    # the same bits again; accumulation adds once; either output may be left out; dx may replace dy
    dx2, dw2, db2 = strided(torch.zeros_like(x), ld), dw.clone(), db.clone()
    assert call(dx2, dw2, db2, True) == 0
    assert torch.equal(dw2, dw + dw) and torch.equal(db2, db + db)
    assert same_bits(dx2, dx)
    assert pool.layer_norm_grad(rows, cols, gs.data_ptr(), ld + 8, xs.data_ptr(), ld, code(dtype), w.data_ptr(), fp.FT_BF16, mean.data_ptr(),
                                rstd.data_ptr(), gs.data_ptr(), ld + 8, 0, db2.data_ptr(), False, ws.data_ptr(), n, stream()) == 0
    assert torch.equal(db2, db) and same_bits(gs, dx)


def test_layer_norm_grad_against_differences(pool):
    rows, cols = 5, 136
    g = gen(7)
    x, w, b, u = randn(g, rows, cols), 1 + 0.1 * randn(g, cols), randn(g, cols), randn(g, rows, cols)
    mean, rstd = torch.empty(2, rows, device="cuda")
    y, dx, (dw, db) = torch.empty_like(x), torch.empty_like(x), torch.empty(2, cols, device="cuda")
    assert pool.layer_norm(rows, cols, x.data_ptr(), cols, fp.FT_F32, w.data_ptr(), b.data_ptr(), fp.FT_F32, EPS, y.data_ptr(), cols,
                           mean.data_ptr(), rstd.data_ptr(), stream()) == 0
    n = pool.layer_norm_grad_workspace(rows, cols)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    assert pool.layer_norm_grad(rows, cols, u.data_ptr(), cols, x.data_ptr(), cols, fp.FT_F32, w.data_ptr(), fp.FT_F32, mean.data_ptr(),
                                rstd.data_ptr(), dx.data_ptr(), cols, dw.data_ptr(), db.data_ptr(), False, ws.data_ptr(), n, stream()) == 0

    def f(x, w, b):  # sum(u y): its gradient is what the call gives for dy = u
        m = x.mean(1, keepdim=True)
        return (u.double() * ((x - m) * (((x - m) ** 2).mean(1, keepdim=True) + EPS) ** -0.5 * w + b)).sum()

    at, h = [t.double() for t in (x, w, b)], 1e-5
    for k, grad in enumerate((dx, dw, db)):
        d = torch.randn(at[k].shape, device="cuda", dtype=torch.float64, generator=g)
        up, down = ([t + s * d if i == k else t for i, t in enumerate(at)] for s in (h, -h))
        slope = (f(*up) - f(*down)) / (2 * h)
        # third derivatives are O(1) here: h^2 of them, and the products' roundings
        assert abs(float(slope - (grad.double() * d).sum())) <= 1e-5 * float((grad.double() * d).abs().sum()) + 1e-7


def test_layer_norm_refusals_and_empty_inputs(pool):
    x = torch.zeros(4, 64, device="cuda")
    w = torch.zeros(64, device="cuda")
    X, W = x.data_ptr(), w.data_ptr()
    ok = dict(rows=4, cols=64, x_ptr=X, ldx=64, dtype=fp.FT_F32, weight_ptr=W, bias_ptr=W, param_dtype=fp.FT_F32, eps=EPS, y_ptr=X, ldy=64)
    assert pool.layer_norm(**ok) == 0
    for bad in (dict(cols=0), dict(ldx=63), dict(ldy=63), dict(dtype=2), dict(param_dtype=9), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(x_ptr=0), dict(y_ptr=0), dict(x_ptr=X + 2), dict(weight_ptr=W + 1), dict(bias_ptr=W + 2)):
        assert pool.layer_norm(**{**ok, **bad}) == INVALID, bad
    assert pool.layer_norm(**{**ok, "cols": (1 << 30) + 1, "ldx": 1 << 31, "ldy": 1 << 31}) == CAPACITY
    assert pool.layer_norm(**{**ok, "rows": 0, "x_ptr": 0, "y_ptr": 0}) == 0
    n = pool.layer_norm_grad_workspace(4, 64)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    dw = torch.full((64,), 3.0, device="cuda")
    ok = dict(rows=4, cols=64, dy_ptr=X, lddy=64, x_ptr=X, ldx=64, dtype=fp.FT_F32, weight_ptr=W, param_dtype=fp.FT_F32, mean_ptr=W, rstd_ptr=W,
              dx_ptr=X, lddx=64, dweight_ptr=dw.data_ptr(), dbias_ptr=0, accumulate=False, ws_ptr=ws.data_ptr(), ws_bytes=n)
    for bad in (dict(cols=0), dict(lddy=1), dict(ldx=1), dict(lddx=1), dict(dtype=7), dict(dy_ptr=0), dict(x_ptr=0), dict(dx_ptr=0), dict(mean_ptr=0),
                dict(rstd_ptr=0), dict(ws_ptr=0), dict(ws_ptr=ws.data_ptr() + 16), dict(dweight_ptr=dw.data_ptr() + 1), dict(dx_ptr=X + 1)):
        assert pool.layer_norm_grad(**{**ok, **bad}) == INVALID, bad
    assert pool.layer_norm_grad(**{**ok, "ws_bytes": n - 1}) == CAPACITY
    torch.cuda.synchronize()
    assert (dw == 3.0).all()
    assert pool.layer_norm_grad(**{**ok, "rows": 0, "accumulate": True, "ws_ptr": 0}) == 0 and (dw == 3.0).all()
    assert pool.layer_norm_grad(**{**ok, "rows": 0, "ws_ptr": 0}) == 0 and (dw == 0.0).all()


# ---- token loss -------------------------------------------------------------------------------------------------

def loss_inputs(seed, rows, hidden, vocab, valid, ldx=None, ldw=None):
    g = gen(seed)
    w = (randn(g, vocab, hidden) * hidden ** -0.5).bfloat16()
    labels = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    x = (randn(g, rows, hidden) + 8 * torch.rand(rows, 1, device="cuda", generator=g) * w[labels].float()).bfloat16()
    labels = torch.where(torch.rand(rows, device="cuda", generator=g) < valid, labels, -100).int()
    return strided(x, ldx or hidden), strided(w, ldw or hidden), labels


def loss_formula(x, w, labels, grad):
    """loss, lse, dx, dw and their error bounds, in 64 bits over the rows that count"""
    rows, hidden = x.shape
    keep = labels != -100
    x6, w6, y = x[keep].double(), w.double(), labels[keep].long()
    z = x6 @ w6.T
    tz = 2 * U * (hidden + 8) * (x6.abs() @ w6.abs().T).amax(1)  # a logit's error
    lse = torch.logsumexp(z, 1)
    picked = z.gather(1, y[:, None])[:, 0]
    # the sum of exponentials: 2 ulp each, vocab / 8 additions in a row at most by one thread, then joins
    t_lse = tz + (32 + x6.shape[0] * 0 + 0.02 * w.shape[0]) * U + 4 * U * (lse.abs() + 16)
    full = lambda v, *s: torch.zeros(rows, *s, dtype=torch.float64, device="cuda").index_copy(0, keep.nonzero()[:, 0], v)  # noqa: E731
    out = dict(loss=full(lse - picked), lse=full(lse), t_loss=full(t_lse + tz + 4 * U * (lse.abs() + picked.abs())), t_lse=full(t_lse))
    if grad is not None:
        gk = grad.double().expand(rows)[keep][:, None]
        d = torch.exp(z - lse[:, None])
        rel = (tz + t_lse)[:, None]
        # bf16 roundings: d over a factor of the row, that factor (chosen so that the label's d needs none), the factor times x
        t_d = d * (rel + 3.03 * B)
        d.scatter_add_(1, y[:, None], torch.full_like(picked, -1.0)[:, None])
        t_d.scatter_(1, y[:, None], (d.gather(1, y[:, None]).abs() * 1.01 * B + rel * (1 + d.gather(1, y[:, None]))))
        d, t_d = d * gk, t_d * gk.abs()
        n = 2 * U * (w.shape[0] + 64)
        out.update(dx=full(d @ w6, hidden), t_dx=full(t_d @ w6.abs() + n * (d.abs() @ w6.abs()), hidden),
                   dw=d.T @ x6, t_dw=t_d.T @ x6.abs() + 2 * U * (rows + 64) * (d.abs().T @ x6.abs()))
    return out


def run_loss(pool, x, w, labels, grad=None, stride=0, dw=None, add=False, ws_bytes=None, fill=0):
    rows, hidden = x.shape
    vocab = w.shape[0]
    loss, lse = torch.full((2, rows), float("nan"), device="cuda")
    dtype = fp.FT_F32 if dw is None or dw.dtype == torch.float32 else fp.FT_BF16
    least, best = pool.token_loss_workspace(rows, hidden, vocab, dw is not None, dtype)
    n = best if ws_bytes is None else ws_bytes(least, best)
    ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
    if dw is None:
        rc = pool.token_loss(rows, hidden, vocab, x.data_ptr(), x.stride(0), w.data_ptr(), w.stride(0), labels.data_ptr(), loss.data_ptr(),
                             lse.data_ptr(), ws.data_ptr(), n, stream())
        return rc, loss, lse, None
    dx = strided(torch.zeros(rows, hidden, device="cuda", dtype=torch.bfloat16), hidden + 8)
    rc = pool.token_loss_grad(rows, hidden, vocab, x.data_ptr(), x.stride(0), w.data_ptr(), w.stride(0), labels.data_ptr(),
                              0 if grad is None else grad.data_ptr(), stride, loss.data_ptr(), lse.data_ptr(), dx.data_ptr(), hidden + 8,
                              dw.data_ptr(), dtype, add, ws.data_ptr(), n, stream())
    return rc, loss, lse, dx


LOSS_SHAPES = [(1, 8, 1, 1.0), (1, 64, 257, 1.0), (2, 8, 1000, 1.0), (3, 72, 63, 1.0), (64, 64, 256, 0.5), (65, 136, 300, 0.7), (127, 128, 511, 1.0),
               (129, 256, 1025, 0.3), (257, 520, 4099, 0.8), (300, 1024, 2048, 0.01), (513, 200, 777, 0.9), (1000, 64, 5003, 0.5)]


@pytest.mark.parametrize("fill", [0, 255])
@pytest.mark.parametrize("shape", LOSS_SHAPES)
def test_token_loss_against_64_bits(pool, shape, fill):
    rows, hidden, vocab, valid = shape
    x, w, labels = loss_inputs(rows * 7 + vocab, rows, hidden, vocab, valid, hidden + 8, hidden + 16)
    e = loss_formula(x, w, labels, torch.ones(1, device="cuda"))
    rc, loss, lse, _ = run_loss(pool, x, w, labels, fill=fill)
    assert rc == 0
    within(loss, e["loss"], e["t_loss"], "loss")
    within(lse, e["lse"], e["t_lse"], "lse")
    for dtype in (torch.float32, torch.bfloat16):
        dw = torch.full((vocab, hidden), float("nan"), device="cuda", dtype=dtype)
        rc, loss2, lse2, dx = run_loss(pool, x, w, labels, dw=dw, fill=fill)
        assert rc == 0
        assert torch.equal(loss2, loss) and torch.equal(lse2, lse)
        within(dx, e["dx"], e["t_dx"] * 1.01 + 1.01 * B * e["dx"].abs() + 1e-30, "dx")
        within(dw, e["dw"], e["t_dw"] * 1.01 + (1.01 * B * e["dw"].abs() if dtype == torch.bfloat16 else 0) + 1e-30, "dw")
        assert (dx[labels == -100] == 0).all()
        gap = torch.as_strided(dx, (rows, 8), (hidden + 8, 1), hidden)
        assert gap.isnan().all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_token_loss_in_pieces_and_accumulating(pool, dtype):
    """Any workspace between the least and the best gives the gradients of the whole; a row gradient per row or one for all."""
    rows, hidden, vocab = 1300, 72, 1111
    x, w, labels = loss_inputs(5, rows, hidden, vocab, 0.6)
    labels[256:512] = -100  # a piece in which nothing counts
    grad = torch.rand(rows, device="cuda", generator=gen(6))
    e = loss_formula(x, w, labels, grad)
    least, best = pool.token_loss_workspace(rows, hidden, vocab, True, code(dtype))
    assert least < best
    for n in (least, (least + best) // 2, best, best + 4096):
        dw = torch.full((vocab, hidden), float("nan"), device="cuda", dtype=dtype)
        rc, loss, lse, dx = run_loss(pool, x, w, labels, grad, 1, dw, ws_bytes=lambda *_: n, fill=255)
        assert rc == 0
        within(loss, e["loss"], e["t_loss"], "loss")
        within(dx, e["dx"], e["t_dx"] * 1.01 + 1.01 * B * e["dx"].abs() + 1e-30, "dx")
        within(dw, e["dw"], e["t_dw"] * 1.01 + 8 * U * e["dw"].abs() + (1.01 * B * e["dw"].abs() if dtype == torch.bfloat16 else 0) + 1e-30, "dw")
        if dtype == torch.float32:
            base = torch.full_like(dw, 0.25)
            assert run_loss(pool, x, w, labels, grad, 1, base, add=True, ws_bytes=lambda *_: n)[0] == 0
            within(base, e["dw"] + 0.25, e["t_dw"] * 1.01 + 16 * U * (e["dw"].abs() + 0.25), "dw added")
    one = torch.full((1,), 0.125, device="cuda")
    e = loss_formula(x, w, labels, one)
    dw = torch.empty((vocab, hidden), device="cuda", dtype=dtype)
    rc, _, _, dx = run_loss(pool, x, w, labels, one, 0, dw)
    assert rc == 0
    within(dx, e["dx"], e["t_dx"] * 1.01 + 1.01 * B * e["dx"].abs() + 1e-30, "dx, one gradient for all rows")


@pytest.mark.parametrize("rows", [1, 70, 400])
def test_rows_without_a_label_reach_nothing(pool, rows):
    """Whatever stands in a masked row, the results are those of the other rows, bit for bit; with no row left, zeros."""
    hidden, vocab = 264, 513
    x, w, labels = loss_inputs(rows, rows, hidden, vocab, 0.5)
    out = []
    for junk in (0.0, float("nan"), float("inf"), -3.3e38):
        xj = x.clone()
        xj[labels == -100] = junk
        dw = torch.full((vocab, hidden), float("nan"), device="cuda")
        rc, loss, lse, dx = run_loss(pool, xj, w, labels, dw=dw)
        assert rc == 0 and (loss[labels == -100] == 0).all() and (lse[labels == -100] == 0).all()
        out.append((loss, lse, dx.contiguous(), dw))
    for o in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, out[0]))
    labels.fill_(-100)
    for dtype in (torch.float32, torch.bfloat16):
        dw = torch.full((vocab, hidden), float("nan"), device="cuda", dtype=dtype)
        rc, loss, lse, dx = run_loss(pool, x, w, labels, dw=dw, fill=255)
        assert rc == 0 and not (loss.any() or lse.any() or dx.any() or dw.any())
    dw = torch.full((vocab, hidden), 2.0, device="cuda")
    assert run_loss(pool, x, w, labels, dw=dw, add=True)[0] == 0 and (dw == 2.0).all()


def test_token_loss_extreme_logits(pool):
    """Logits whose exponentials alone would overflow or vanish, a tile of the vocabulary far below another, equal logits,
    and rows that are not finite."""
    hidden, vocab = 64, 1200
    w = torch.zeros(vocab, hidden, device="cuda", dtype=torch.bfloat16)
    w[:, 0] = torch.linspace(-1, 1, vocab, device="cuda")
    x = torch.zeros(8, hidden, device="cuda", dtype=torch.bfloat16)
    x[:, 0] = torch.tensor([0.0, 1.0, 100.0, -100.0, 3000.0, -3000.0, 1e30, -1e30])
    labels = torch.tensor([0, 1199, 1199, 0, 0, 600, 1199, 3], device="cuda", dtype=torch.int32)
    e = loss_formula(x, w, labels, torch.ones(1, device="cuda"))
    dw = torch.empty(vocab, hidden, device="cuda")
    rc, loss, lse, dx = run_loss(pool, x, w, labels, dw=dw)
    assert rc == 0
    within(loss, e["loss"], e["t_loss"], "loss")
    within(lse, e["lse"], e["t_lse"], "lse")
    small = x[:6]
    e = loss_formula(small, w, labels[:6], torch.ones(1, device="cuda"))
    rc, loss, lse, dx = run_loss(pool, small, w, labels[:6].contiguous(), dw=dw)
    within(dx, e["dx"], e["t_dx"] * 1.01 + 1.01 * B * e["dx"].abs() + 1e-30, "dx")
    within(dw, e["dw"], e["t_dw"] * 1.01 + 1e-30, "dw")
    bad = small.clone()
    bad[2, 5] = float("nan")
    rc, loss, lse, dx = run_loss(pool, bad, w, labels[:6].contiguous(), dw=dw)
    assert rc == 0 and loss[2].isnan() and lse[2].isnan() and dx[2].isnan().all()
    assert loss[[0, 1, 3, 4, 5]].isfinite().all() and dx[[0, 1, 3, 4, 5]].isfinite().all()


def test_token_loss_grad_against_differences(pool):
    rows, hidden, vocab = 21, 64, 300
    x, w, labels = loss_inputs(3, rows, hidden, vocab, 0.8)
    g = gen(4)
    c = torch.rand(rows, device="cuda", generator=g)
    dw = torch.empty(vocab, hidden, device="cuda")
    rc, loss, lse, dx = run_loss(pool, x, w, labels, c, 1, dw)
    assert rc == 0
    e = loss_formula(x, w, labels, c)

    def f(x, w):
        z = x @ w.T
        l = torch.logsumexp(z, 1) - z.gather(1, labels.clamp_min(0).long()[:, None])[:, 0]
        return (torch.where(labels >= 0, l, 0.0) * c.double()).sum()

    at, h = [x.double(), w.double()], 1e-4
    for k, (grad, bound) in enumerate(((dx, e["t_dx"] + B * e["dx"].abs()), (dw, e["t_dw"]))):
        for _ in range(4):
            d = torch.randn(at[k].shape, device="cuda", dtype=torch.float64, generator=g)
            up, down = ([t + s * d if i == k else t for i, t in enumerate(at)] for s in (h, -h))
            slope = (f(*up) - f(*down)) / (2 * h)
            # the central difference is off by h^2 times third derivatives, below 1e-3 of the directions' length here
            assert abs(float(slope - (grad.double() * d).sum())) <= float((bound * d.abs()).sum()) + 1e-3 * h * float(d.abs().sum())


def test_bad_labels_are_reported_and_skipped(pool):
    rows, hidden, vocab = 90, 64, 128
    x, w, labels = loss_inputs(8, rows, hidden, vocab, 1.0)
    masked = labels.clone()
    masked[[17, 40, 77]] = -100
    labels[17], labels[40], labels[77] = 128, -1, 2 ** 31 - 1
    dw, dm = torch.empty(2, vocab, hidden, device="cuda")
    assert pool.status() == (0, 0)
    a = run_loss(pool, x, w, labels, dw=dw)
    assert pool.status() == (BAD_ID, 17) and pool.status() == (0, 0)
    b = run_loss(pool, x, w, masked, dw=dm)
    assert a[0] == b[0] == 0 and torch.equal(dw, dm) and all(torch.equal(s.contiguous(), t.contiguous()) for s, t in zip(a[1:], b[1:]))
    assert pool.status() == (0, 0)


def test_token_loss_refusals_and_empty_inputs(pool):
    rows, hidden, vocab = 10, 64, 100
    x, w, labels = loss_inputs(1, rows, hidden, vocab, 1.0)
    loss, dw = torch.zeros(rows, device="cuda"), torch.full((vocab, hidden), 7.0, device="cuda")
    least, best = pool.token_loss_workspace(rows, hidden, vocab, True, fp.FT_F32)
    ws = torch.empty(best, dtype=torch.uint8, device="cuda")
    X, W, L, D = x.data_ptr(), w.data_ptr(), loss.data_ptr(), dw.data_ptr()
    ok = dict(rows=rows, hidden=hidden, vocab=vocab, x_ptr=X, ldx=hidden, w_ptr=W, ldw=hidden, labels_ptr=labels.data_ptr(), loss_ptr=L, lse_ptr=L,
              ws_ptr=ws.data_ptr(), ws_bytes=best)
    more = dict(grad_loss_ptr=0, grad_stride=0, dx_ptr=X, lddx=hidden, dw_ptr=D, dw_dtype=fp.FT_F32, accumulate=False)
    both = (dict(hidden=0), dict(hidden=60), dict(vocab=0), dict(x_ptr=0), dict(x_ptr=X + 2), dict(ldx=56), dict(ldx=65), dict(w_ptr=0), dict(w_ptr=W + 8),
            dict(ldw=32), dict(ldw=68), dict(labels_ptr=0), dict(labels_ptr=labels.data_ptr() + 1), dict(loss_ptr=0), dict(lse_ptr=0), dict(ws_ptr=0),
            dict(ws_ptr=ws.data_ptr() + 128))
    for bad in both:
        assert pool.token_loss(**{**ok, **bad}) == INVALID, bad
        assert pool.token_loss_grad(**{**ok, **more, **bad}) == INVALID, bad
    for bad in (dict(grad_loss_ptr=L + 2), dict(grad_stride=2), dict(dx_ptr=0), dict(dx_ptr=X + 4), dict(lddx=63), dict(dw_ptr=0), dict(dw_ptr=D + 4),
                dict(dw_dtype=5), dict(dw_dtype=fp.FT_BF16, accumulate=True)):
        assert pool.token_loss_grad(**{**ok, **more, **bad}) == INVALID, bad
    assert pool.token_loss_grad(**{**ok, **more, "ws_bytes": least - 1}) == CAPACITY
    assert pool.token_loss(**{**ok, "rows": 1 << 31}) == CAPACITY and pool.token_loss(**{**ok, "vocab": 1 << 31}) == CAPACITY
    torch.cuda.synchronize()
    assert (dw == 7.0).all()
    assert pool.token_loss(**{**ok, "rows": 0, "x_ptr": 0, "ws_ptr": 0}) == 0
    assert pool.token_loss_grad(**{**ok, **more, "rows": 0, "accumulate": True, "ws_ptr": 0}) == 0 and (dw == 7.0).all()
    assert pool.token_loss_grad(**{**ok, **more, "rows": 0, "ws_ptr": 0}) == 0 and (dw == 0.0).all()


def test_operators_on_another_stream_and_in_a_graph(pool):
    """Work queued on a side stream is seen in stream order, and a captured step replays on new inputs."""
    rows, hidden, vocab = 200, 128, 999
    x, w, labels = loss_inputs(11, rows, hidden, vocab, 0.7)
    x2, _, labels2 = loss_inputs(12, rows, hidden, vocab, 0.9)
    dw, dw1, dw2 = torch.empty(3, vocab, hidden, device="cuda")
    first, second = run_loss(pool, x, w, labels, dw=dw1), run_loss(pool, x2, w, labels2, dw=dw2)
    torch.cuda.synchronize()
    loss, lse = torch.empty(2, rows, device="cuda")
    dx = torch.empty(rows, hidden, device="cuda", dtype=torch.bfloat16)
    n = pool.token_loss_workspace(rows, hidden, vocab, True, fp.FT_F32)[1]
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    xin, lin = torch.zeros_like(x), labels.clone()
    side = torch.cuda.Stream()

    def step(st):
        assert pool.token_loss_grad(rows, hidden, vocab, xin.data_ptr(), xin.stride(0), w.data_ptr(), w.stride(0), lin.data_ptr(), 0, 0, loss.data_ptr(),
                                    lse.data_ptr(), dx.data_ptr(), hidden, dw.data_ptr(), fp.FT_F32, False, ws.data_ptr(), n, st) == 0

    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        xin.copy_(x)
        step(side.cuda_stream)
    side.synchronize()
    assert torch.equal(loss, first[1]) and torch.equal(dx, first[3].contiguous()) and torch.equal(dw, dw1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream().cuda_stream)
    xin.copy_(x2)
    lin.copy_(labels2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(loss, second[1]) and torch.equal(dx, second[3].contiguous()) and torch.equal(dw, dw2)


# ---- AdamW ------------------------------------------------------------------------------------------------------

CFG = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8)


def pack8(val, floor):
    """The 8-bit form of a flat fp32 tensor: float8 values and a scale per 256, from the definition (on the CPU)."""
    n = val.numel()
    b = torch.nn.functional.pad(val, (0, -n % 256)).view(-1, 256)
    top = b.abs().amax(1)
    scale = torch.where(top > 0, torch.exp2(torch.ceil(torch.log2(top.double() / 448)).clamp(-100, 100)).float(), 0.0)
    q = torch.where(scale[:, None] > 0, b / scale[:, None], 0.0)
    if floor:
        q = torch.where((q > 0) & (q < 2.0 ** -9), 2.0 ** -9, q)
    return q.view(-1)[:n].to(torch.float8_e4m3fn), scale


def unpack8(q, scale):
    return (torch.nn.functional.pad(q.float(), (0, -q.numel() % 256)).view(-1, 256) * scale[:, None]).view(-1)[: q.numel()]


class AdamwCase:
    """One tensor on the GPU and its fp32 reference on the CPU, each operation rounded by itself."""

    def __init__(self, seed, n, param, grad, bits, copy, shift=0, zero=False):
        g = torch.Generator().manual_seed(seed)
        self.n, self.bits, self.wd = n, bits, 0.1 * (seed % 3)
        scale = torch.exp(2 * torch.randn(n, generator=g))
        self.p = torch.randn(n, generator=g).to(param)
        self.g = (scale * torch.randn(n, generator=g)).to(grad)
        m, r = scale * torch.randn(n, generator=g), scale * torch.rand(n, generator=g)
        if zero:
            m, r = torch.zeros(n), torch.zeros(n)
        if bits == 32:
            self.state = [m, r * r]
        else:
            (m, ms), (r, rs) = pack8(m, False), pack8(r, True)
            self.state = [m, r, ms, rs]
        self.copy = torch.zeros(n, dtype=torch.bfloat16) if copy else None
        self.dev = [self.place(t, shift) for t in (self.p, self.g, *self.state, *([self.copy] if copy else []))]

    @staticmethod
    def place(t, shift):
        raw = torch.full((t.numel() * t.element_size() + 512,), 0x5A, dtype=torch.uint8, device="cuda")
        at = raw[shift * t.element_size():][: t.numel() * t.element_size()]
        at.copy_(t.view(torch.uint8).cuda())
        return raw, at, t.dtype

    def host(self, i):
        raw, at, dtype = self.dev[i]
        return at.cpu().view(dtype)

    def tensor(self):
        ptr = [at.data_ptr() for _, at, _ in self.dev]
        s8 = self.bits == 8
        return fp.AdamwTensor(param=ptr[0], grad=ptr[1], m=ptr[2], v=ptr[3], m_scale=ptr[4] if s8 else None, v_scale=ptr[5] if s8 else None,
                              copy=ptr[-1] if self.copy is not None else None, n=self.n, weight_decay=self.wd, param_dtype=code(self.p.dtype),
                              grad_dtype=code(self.g.dtype), state_bits=self.bits)

    def step(self, t, gscale=1.0):
        f = lambda x: torch.tensor(x, dtype=torch.float64).float()  # noqa: E731
        g = self.g.float() * f(gscale)
        if self.bits == 8:
            m, r = unpack8(self.state[0], self.state[2]), unpack8(self.state[1], self.state[3])
            v = r * r
        else:
            m, v = self.state
        m = f(CFG["beta1"]) * m + f(1 - CFG["beta1"]) * g
        v = f(CFG["beta2"]) * v + f(1 - CFG["beta2"]) * (g * g)
        r = v.sqrt()
        if self.bits == 8:
            (a, sa), (b, sb) = pack8(m, False), pack8(r, True)
            self.state = [a, b, sa, sb]
        else:
            self.state = [m, v]
        m6, r6, p6 = m.double(), r.double(), self.p.double()
        step = CFG["lr"] / (1 - CFG["beta1"] ** t) * m6 / (r6 / (1 - CFG["beta2"] ** t) ** 0.5 + CFG["eps"])
        self.exp = p6 * (1 - CFG["lr"] * self.wd) - step
        # the step's factors and quotient: eight roundings; the parameter's own product and difference: three
        self.bound = 16 * U * step.abs() + 4 * U * (p6.abs() + self.exp.abs()) + 1e-37
        if self.p.dtype == torch.bfloat16:
            self.bound = self.bound + 1.01 * B * self.exp.abs()

    def check(self):
        n_state = len(self.state)
        for i, s in enumerate(self.state):
            assert torch.equal(self.host(2 + i).view(torch.uint8), s.view(torch.uint8)), f"state {i} of n={self.n}"
        p = self.host(0)
        bad = ~((p.double() - self.exp).abs() <= self.bound)
        assert not bad.any(), f"{int(bad.sum())} parameters of n={self.n}"
        if self.copy is not None:
            c = self.host(2 + n_state).double()
            assert ((c - p.double()).abs() <= B * 1.01 * p.double().abs()).all()
        for raw, at, _ in self.dev:  # nothing beside the arrays was written
            lo = at.data_ptr() - raw.data_ptr()
            assert (raw[:lo] == 0x5A).all() and (raw[lo + at.numel():] == 0x5A).all()
        self.p = p

    def grad_again(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.g = torch.randn(self.n, generator=g).to(self.g.dtype)
        self.dev[1][1].copy_(self.g.view(torch.uint8).cuda())


TYPES = [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("types", TYPES)
def test_adamw_against_the_formula(pool, types, bits):
    """Sizes around a block and a chunk, aligned and shifted starts, all in one list; three steps."""
    sizes = [1, 2, 7, 255, 256, 257, 2047, 2048, 2049, 5000, 40001]
    cases = [AdamwCase(17 * i + s, n, *types, bits, copy=i % 2 == 0, shift=s) for i, n in enumerate(sizes) for s in (0, 1, 8)]
    scale = torch.full((1,), 0.5, device="cuda")
    arr = (fp.AdamwTensor * len(cases))(*[c.tensor() for c in cases])
    for t in (1, 2, 3):
        cfg = fp.AdamwConfig(**CFG, step=t, grad_scale=scale.data_ptr() if t == 2 else None)
        assert pool.adamw_step(arr, cfg, stream()) == 0
        torch.cuda.synchronize()
        for i, c in enumerate(cases):
            c.step(t, 0.5 if t == 2 else 1.0)
            c.check()
            c.grad_again(1000 * t + i)


def test_adamw_many_tensors_of_mixed_kinds_and_empty_ones(pool):
    kinds = [(p, g, b) for p, g in TYPES for b in (32, 8)]
    cases = [AdamwCase(i, 1 + (i * 37) % 600, *kinds[i % 8][:2], kinds[i % 8][2], copy=i % 5 == 0, shift=i % 3, zero=i % 7 == 0) for i in range(700)]
    empty = fp.AdamwTensor(n=0, state_bits=8, param_dtype=fp.FT_F32, grad_dtype=fp.FT_F32)
    arr = []
    for i, c in enumerate(cases):
        arr.append(c.tensor())
        if i % 50 == 0:
            arr.append(empty)
    assert pool.adamw_step(arr, fp.AdamwConfig(**CFG, step=9), stream()) == 0
    torch.cuda.synchronize()
    for c in cases:
        c.step(9)
        c.check()
    assert pool.adamw_step([], fp.AdamwConfig(**CFG, step=1), stream()) == 0
    assert pool.adamw_step([empty], fp.AdamwConfig(**CFG, step=1), stream()) == 0


def test_adamw_8_bit_blocks_that_are_not_finite_zero_or_tiny(pool):
    n = 256 * 6 + 40
    c = AdamwCase(3, n, torch.float32, torch.float32, 8, False, zero=True)
    g = torch.randn(n, generator=torch.Generator().manual_seed(2))
    g[256:512] = 0                                   # nothing: scale and values stay zero, the parameters only decay
    g[512:768] *= 1e-18                              # v = g^2 is a subnormal fp32 number
    g[768:1024] = 0
    g[800], g[801] = 1.0, 1e-6                       # a positive r far below the block's scale keeps the smallest value
    g[1024 + 9] = float("nan")
    g[1280 + 7] = float("inf")
    c.g = g
    c.dev[1][1].copy_(g.view(torch.uint8).cuda())
    assert pool.adamw_step([c.tensor()], fp.AdamwConfig(**CFG, step=1), stream()) == 0
    torch.cuda.synchronize()
    m, r, ms, rs = (c.host(i) for i in (2, 3, 4, 5))
    p0 = c.p
    c.step(1)
    clean = [0, 1, 2, 3, 6]
    for got, exp in ((ms, c.state[2]), (rs, c.state[3])):
        assert torch.equal(got[clean], exp[clean]) and got[[4, 5]].isnan().all()
    for got, exp in ((m, c.state[0]), (r, c.state[1])):
        for b in clean:
            assert torch.equal(got[256 * b:256 * b + 256].view(torch.uint8), exp[256 * b:256 * b + 256].view(torch.uint8)), b
    assert ms[1] == 0 and rs[1] == 0 and float(r[801]) == 2.0 ** -9
    p = c.host(0)
    within(p[256:512].double(), p0[256:512].double() * (1 - CFG["lr"] * c.wd), 4 * U * p0[256:512].double().abs(), "decay alone")
    assert p[1024 + 9].isnan() and p[1024:1024 + 9].isfinite().all()


def test_adamw_refusals(pool):
    c = AdamwCase(1, 300, torch.float32, torch.float32, 8, True)
    before = [c.host(i).view(torch.uint8).clone() for i in range(len(c.dev))]

    def call(cfg=None, **tensor):
        t = c.tensor()
        for k, v in tensor.items():
            setattr(t, k, v)
        return pool.adamw_step([c.tensor(), t], fp.AdamwConfig(**{**CFG, "step": 1, **(cfg or {})}), stream())

    nan = float("nan")
    for bad in (dict(lr=nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan), dict(eps=-1.0), dict(eps=float("inf")), dict(step=0),
                dict(grad_scale=2)):
        assert call(cfg=bad) == INVALID, bad
    t = c.tensor()
    for bad in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(m_scale=None), dict(v_scale=None), dict(param=t.param + 2),
                dict(grad=t.grad + 1), dict(m_scale=t.m_scale + 2), dict(copy=t.copy + 1), dict(param_dtype=2), dict(grad_dtype=3), dict(state_bits=16),
                dict(weight_decay=nan)):
        assert call(**bad) == INVALID, bad
    assert call(state_bits=32, m=t.m + 1) == INVALID
    assert call(n=(1 << 40) + 1) == CAPACITY
    assert fp.lib().pool_adamw_step(pool.h, None, 1, ctypes.byref(fp.AdamwConfig(**CFG, step=1)), None) == INVALID
    assert fp.lib().pool_adamw_step(pool.h, None, 0, None, None) == INVALID
    torch.cuda.synchronize()
    for i, b in enumerate(before):
        assert torch.equal(c.host(i).view(torch.uint8), b)


def test_a_new_pool_counts_its_launches():
    p = fp.Pool(fp.PoolConfig(page_bytes=4096, hbm_pages=1, max_text_tokens=1024, hidden=8, max_samples=1, max_spans_per_sample=1,
                              max_pages_per_span=1, max_seq_len=1))
    assert p.rc == 0
    x = torch.zeros(4, 64, device="cuda")
    n0 = p.stats()["gpu_launches"]
    assert p.layer_norm(4, 64, x.data_ptr(), 64, fp.FT_F32, 0, 0, fp.FT_F32, EPS, x.data_ptr(), 64, 0, 0, stream()) == 0
    assert p.stats()["gpu_launches"] == n0 + 1
    torch.cuda.synchronize()
    p.destroy()
