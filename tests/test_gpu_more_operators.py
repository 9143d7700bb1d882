"""Rotary positions, the root-mean-square norm, the gradients' norm and token log probabilities on the GPU, against plain 64-bit
implementations of their formulas.  Every tolerance is an error bound worked out from the formula: U is fp32's unit roundoff, B
bf16's, E8 e4m3's; a sum of n fp32 terms in any order is off by at most n U times the sum of the terms' magnitudes (2 U for the tensor
cores, whose additions may truncate)."""
import math

import numpy as np
import pytest
import torch

from paper_2606_23087_b200 import binding as fp

pytestmark = pytest.mark.gpu

U, B, E8 = 2.0 ** -24, 2.0 ** -8, 2.0 ** -4
INVALID, BAD_ID, CAPACITY, TIMEOUT = -1, -9, -11, -13
TYPES = [torch.bfloat16, torch.float32]


def new_pool():
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    p = fp.Pool(fp.PoolConfig(page_bytes=4096, hbm_pages=1, max_text_tokens=1024, hidden=8, max_samples=1, max_spans_per_sample=1,
                              max_pages_per_span=1, max_seq_len=1))
    assert p.rc == 0
    return p


@pytest.fixture(scope="module")
def pool():
    p = new_pool()
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


def code(t):
    return fp.FT_BF16 if t == torch.bfloat16 else fp.FT_F32


def half_step(t):
    return B if t == torch.bfloat16 else U


def strided(t, ld, shift=0):
    """A copy of the matrix with row stride ld, `shift` elements into its buffer, the rest NaN (0x7F where the type has 8 bits)."""
    rows, cols = t.shape
    if t.element_size() == 1:
        buf = torch.full((rows * ld + shift + 64,), 0x7F, dtype=torch.uint8, device="cuda").view(t.dtype)
    else:
        buf = torch.full((rows * ld + shift + 64,), float("nan"), dtype=t.dtype, device="cuda")
    view = torch.as_strided(buf, (rows, cols), (ld, 1), shift)
    view.copy_(t)
    return view


def beside(t):
    """The elements between the rows of a strided matrix."""
    rows, cols = t.shape
    return torch.as_strided(t, (rows, t.stride(0) - cols), (t.stride(0), 1), t.storage_offset() + cols)


def bits(t):
    return t.contiguous().view(torch.uint8)


def within(got, exp, bound, what):
    got, exp = got.double(), exp.double()
    bad = ~((got - exp).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float(((got - exp).abs() / bound).max()):.3g} times it"


# ---- rotary -----------------------------------------------------------------------------------------------------

def turned(x, pos, freqs, axes, interleaved, inverse):
    """The formula on [rows, heads, dim], angles reduced in extended precision, and the magnitudes that its bound scales with."""
    rows, heads, dim = x.shape
    n = len(freqs)
    p = pos.cpu().numpy().astype(np.longdouble)
    turns = np.stack([p[axes[i]] * (np.longdouble(freqs[i]) / (2 * np.longdouble("3.14159265358979323846264338327950288"))) for i in range(n)], 1)
    angle = torch.from_numpy(((turns - np.rint(turns)) * 2 * np.longdouble("3.14159265358979323846264338327950288")).astype(np.float64)).cuda()
    if inverse:
        angle = -angle
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    y, mag = x.double().clone(), torch.zeros_like(x, dtype=torch.float64)
    first = torch.arange(n, device="cuda") * (2 if interleaved else 1)
    second = first + (1 if interleaved else n)
    a, b = x[..., first].double(), x[..., second].double()
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    mag[..., first] = mag[..., second] = a.abs() + b.abs()
    return y, mag


ROTARY = [  # rows, heads of each tensor, head_dim, pairs, interleaved
    (1, (1,), 2, 1, False), (1, (28, 4), 128, 64, False), (3, (5, 1), 96, 32, True), (7, (2, 2, 1, 1, 3), 64, 32, False), (130, (3,), 11, 5, True),
    (33, (2, 1), 80, 40, False), (600, (32, 8), 128, 64, True), (5, (300,), 16, 8, False), (9, (1, 2), 512, 256, False), (4, (2,), 512, 3, True),
    (1201, (1,), 130, 60, False), (2, (1,), 24, 4, False)]


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", ROTARY)
def test_rotary_against_64_bits(pool, shape, dtype, inverse):
    rows, heads, dim, pairs, interleaved = shape
    g = gen(rows * 131 + dim)
    rng = np.random.default_rng(rows + dim)
    freqs = 1e4 ** (-np.arange(pairs) / pairs)
    axes = rng.integers(0, 3, pairs).astype(np.uint8)
    pos = torch.randint(0, 1 << 20, (3, rows + 5), device="cuda", generator=g, dtype=torch.int32)
    pos[:, 0] = torch.tensor([2 ** 31 - 1, -7, 0])
    pos[2, rows // 2] = -2 ** 31
    total = sum(heads)
    src = strided((randn(g, rows, total * dim) * 3).to(dtype), total * dim + 16)  # the heads of all tensors in one row, and 16 more elements
    cfg = fp.rotary_config(freqs, axes, dim, interleaved, inverse)

    def tensors(dst, dst_row, dst_head, shift=lambda at: at):
        out, at = [], 0
        for h in heads:
            out.append(fp.RotaryTensor(src=src.data_ptr() + at * dim * src.element_size(), dst=dst.data_ptr() + shift(at) * dst.element_size(),
                                       src_row=src.stride(0), src_head=dim, dst_row=dst_row, dst_head=dst_head, heads=h, dtype=code(dtype)))
            at += h
        return out

    expect, mag = turned(src.view(rows, total, dim) if src.is_contiguous() else src.reshape(rows, total, dim), pos[:, :rows], freqs, axes, interleaved, inverse)
    # sine and cosine 2 ulp, their argument 2^-25 of pi, two products and a sum; then one rounding
    bound = 10 * U * mag + 1.01 * half_step(dtype) * expect.abs() + 1e-38
    # rows apart
    dst = strided(torch.zeros(rows, total * dim, dtype=dtype, device="cuda"), total * dim + 8)
    assert pool.rotary(rows, pos.data_ptr(), rows + 5, cfg, tensors(dst, dst.stride(0), dim, lambda at: at * dim), stream()) == 0
    within(dst.reshape(rows, total, dim), expect, bound, "rows apart")
    assert beside(dst).isnan().all()
    rest = [i for i in range(dim) if i >= 2 * pairs]
    assert torch.equal(bits(dst.reshape(rows, total, dim)[..., rest]), bits(src.reshape(rows, total, dim)[..., rest]))
    # heads apart
    apart = torch.full((total, rows, dim), float("nan"), dtype=dtype, device="cuda")
    assert pool.rotary(rows, pos.data_ptr(), rows + 5, cfg, tensors(apart, dim, rows * dim, lambda at: at * rows * dim), stream()) == 0
    assert torch.equal(bits(apart.transpose(0, 1)), bits(dst.reshape(rows, total, dim)))
    # in place
    assert pool.rotary(rows, pos.data_ptr(), rows + 5, cfg, [fp.RotaryTensor(src=t.src, dst=t.src, src_row=t.src_row, src_head=dim, dst_row=t.src_row,
                                                                            dst_head=dim, heads=t.heads, dtype=t.dtype)
                                                            for t in tensors(dst, 0, 0)], stream()) == 0
    assert torch.equal(bits(src), bits(dst))
    assert beside(src).isnan().all()


def test_rotary_off_16_bytes_one_axis_and_mixed_types(pool):
    """The same values from operands that allow no wide access; positions of one axis; tensors of both types in one call."""
    rows, dim = 37, 64
    g = gen(3)
    freqs = 1e6 ** (-np.arange(32) / 32)
    pos = torch.arange(rows, device="cuda", dtype=torch.int32) + 70000
    x = strided(randn(g, rows, 2 * dim).bfloat16(), 2 * dim + 3, 1)
    f = strided(randn(g, rows, dim), dim)
    y, z = strided(torch.zeros_like(x), 2 * dim + 1, 3), torch.zeros_like(f)
    cfg = fp.rotary_config(freqs, None, dim)
    both = [fp.RotaryTensor(src=x.data_ptr(), dst=y.data_ptr(), src_row=x.stride(0), src_head=dim, dst_row=y.stride(0), dst_head=dim, heads=2, dtype=fp.FT_BF16),
            fp.RotaryTensor(src=f.data_ptr(), dst=z.data_ptr(), src_row=dim, src_head=dim, dst_row=dim, dst_head=dim, heads=1, dtype=fp.FT_F32)]
    assert pool.rotary(rows, pos.data_ptr(), 0, cfg, both, stream()) == 0
    for got, src, h, t in ((y, x, 2, torch.bfloat16), (z, f, 1, torch.float32)):
        e, mag = turned(src.reshape(rows, h, dim), pos[None], freqs, [0] * 32, False, False)
        within(got.reshape(rows, h, dim), e, 10 * U * mag + 1.01 * half_step(t) * e.abs() + 1e-38, str(t))
    assert beside(y).isnan().all()


def test_rotary_turned_back_is_the_transpose(pool):
    """<R x, u> = <x, R^T u>, which is the gradient's definition for a linear map, and R^T R x = x."""
    rows, heads, dim = 50, 3, 48
    g = gen(11)
    pos = torch.randint(0, 5000, (3, rows), device="cuda", generator=g, dtype=torch.int32)
    freqs, axes = 1e4 ** (-np.arange(20) / 20), np.arange(20) % 3
    x, u = randn(g, rows, heads, dim), randn(g, rows, heads, dim)

    def turn(v, inverse):
        out = torch.empty_like(v)
        t = fp.RotaryTensor(src=v.data_ptr(), dst=out.data_ptr(), src_row=heads * dim, src_head=dim, dst_row=heads * dim, dst_head=dim, heads=heads, dtype=fp.FT_F32)
        assert pool.rotary(rows, pos.data_ptr(), rows, fp.rotary_config(freqs, axes, dim, True, inverse), [t], stream()) == 0
        return out
    y, back = turn(x, False), turn(u, True)
    one, two = (y.double() * u.double()).sum(), (x.double() * back.double()).sum()
    assert abs(float(one - two)) <= 2 * 20 * U * float((x.abs().double() + 1).sum() * 8)
    within(turn(y, True), x, 40 * U * (x.abs() + 8), "there and back")


def test_rotary_refusals_and_empty_inputs(pool):
    x = torch.zeros(4, 2, 8, device="cuda")
    pos = torch.zeros(3, 4, device="cuda", dtype=torch.int32)
    X, P = x.data_ptr(), pos.data_ptr()
    tensor = dict(src=X, dst=X, src_row=16, src_head=8, dst_row=16, dst_head=8, heads=2, dtype=fp.FT_F32)

    def call(rows=4, pos_ptr=P, pos_ld=4, freqs=(1.0, 0.5), axes=(0, 2), dim=8, n=None, **change):
        return pool.rotary(rows, pos_ptr, pos_ld, fp.rotary_config(freqs, axes, dim), [fp.RotaryTensor(**{**tensor, **change})], stream())

    assert call() == 0
    for bad in (dict(pos_ptr=0), dict(pos_ptr=P + 2), dict(pos_ld=3), dict(freqs=(1.0, math.nan)), dict(freqs=(math.inf, 1.0)), dict(freqs=(1.0, 1e10)),
                dict(axes=(0, 3)), dict(dim=3), dict(src=0), dict(dst=0), dict(src=X + 2, dst=X + 2), dict(dtype=2), dict(dst_row=20),
                dict(dst=X + 512, dst_head=4), dict(dst=X + 512, dst_row=8), dict(dst=X + 512, dst_row=12)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(dim=513), dict(heads=8193), dict(rows=1 << 31)):
        assert call(**bad) == CAPACITY, bad
    assert call(axes=None, pos_ld=0) == 0     # one axis needs no stride
    assert call(rows=0, pos_ptr=0, src=0, dst=0) == 0
    assert call(heads=0, src=0, dst=0) == 0
    cfg = fp.rotary_config((1.0,), None, 8)
    assert pool.rotary(4, P, 4, cfg, [], stream()) == 0
    cfg.freq = None
    assert pool.rotary(4, P, 4, cfg, [fp.RotaryTensor(**tensor)], stream()) == INVALID
    cfg = fp.rotary_config((1.0,), None, 8)
    cfg.pairs = 0
    assert pool.rotary(4, P, 4, cfg, [fp.RotaryTensor(**tensor)], stream()) == INVALID
    torch.cuda.synchronize()
    assert (x == 0).all()


# ---- root-mean-square norm --------------------------------------------------------------------------------------

EPS = 1e-6
SHAPES = [(1, 1), (3, 1), (1, 8), (5, 31), (33, 64), (7, 129), (300, 1000), (257, 1023), (64, 1024), (1, 3584), (150, 3584), (700, 4096),
          (9, 8192), (12, 8191), (5, 8200), (400, 5000), (4, 12296), (3, 16384), (3, 20001), (2, 20480)]


def rms_formula(x, res, w):
    s = x.double() + (0 if res is None else res.double())
    rstd = ((s * s).mean(1, keepdim=True) + EPS) ** -0.5
    return s, rstd, s * rstd * w.double()


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_rms_norm_against_64_bits(pool, shape, dtype, residual):
    rows, cols = shape
    g = gen(rows * 10007 + cols)
    x = (randn(g, rows, cols) * torch.exp(randn(g, rows, 1))).to(dtype)
    res = randn(g, rows, cols).to(dtype) if residual else None
    w = (1 + 0.1 * randn(g, cols)).to(torch.bfloat16 if cols % 2 else torch.float32)
    ld = cols + 3 if cols % 2 else cols
    xs, rs = strided(x, ld), strided(res, ld) if residual else None
    y, total = strided(torch.zeros_like(x), ld + 8), strided(torch.zeros_like(x), ld)
    groups = -(-cols // 128)
    q, scale = strided(torch.zeros(rows, cols, dtype=torch.uint8, device="cuda"), ld + 8), strided(torch.zeros(rows, groups, device="cuda"), groups + 1)
    rstd = torch.empty(rows, device="cuda")

    def call(y, q):
        return pool.rms_norm(rows, cols, xs.data_ptr(), ld, rs.data_ptr() if residual else 0, ld, code(dtype), w.data_ptr(), code(w.dtype), EPS,
                             total.data_ptr(), ld, y, ld + 8, q, ld + 8, scale.data_ptr() if q else 0, groups + 1, rstd.data_ptr(), stream())

    assert call(y.data_ptr(), 0) == 0
    s6, r6, e6 = rms_formula(x, res, w)
    rounding = half_step(dtype) * 1.001
    within(total, s6, rounding * s6.abs(), "sum")
    within(rstd[:, None], r6, 40 * U * r6, "rstd")   # 64 roundings in a row's sum at most, halved by the root, and the root's 2 ulp
    within(y, e6, (44 * U + rounding) * e6.abs() + 1e-38, "y")
    assert beside(y).isnan().all() and (beside(total).isnan().all() if ld > cols else True)
    # in 8 bits, alone and beside y: the scale is the group's largest magnitude over 448, a value off by half a step of the format
    for both in (False, True):
        y.fill_(0)
        assert call(y.data_ptr() if both else 0, q.data_ptr()) == 0
        if both:   # (another kernel may have taken the sums where there are 8 bits)
            within(y, e6, (44 * U + rounding) * e6.abs() + 1e-38, "y beside q")
        else:
            assert (y == 0).all()
        top = torch.nn.functional.pad(e6.abs(), (0, -cols % 128)).view(rows, groups, 128).amax(2)
        within(scale, top / 448, 50 * U * top / 448 + 1e-38, "scale")
        wide = scale.double().repeat_interleave(128, 1)[:, :cols]
        got = q.contiguous().view(torch.float8_e4m3fn).double() * wide
        within(got, e6, 1.01 * E8 * e6.abs() + wide * 2.0 ** -10 * 1.01 + 60 * U * e6.abs(), "q")
        assert (beside(q) == 0x7F).all() and beside(scale).isnan().all()


@pytest.mark.parametrize("cols", [1, 40, 1023, 3584, 9000, 20000])
def test_rms_norm_keeps_bad_rows_to_themselves_and_works_in_place(pool, cols):
    g = gen(cols)
    x, res = randn(g, 6, cols).bfloat16(), randn(g, 6, cols).bfloat16()
    x[1, cols // 2] = float("nan")
    x[3, 0] = float("inf")
    x[4], res[4] = 2.5, -2.5  # a row of zeros
    w = randn(g, cols).bfloat16()
    y, total = torch.empty_like(x), torch.empty_like(x)
    groups = -(-cols // 128)
    q, scale = torch.empty(6, cols, dtype=torch.uint8, device="cuda"), torch.empty(6, groups, device="cuda")

    def call(x, res, total, y):
        return pool.rms_norm(6, cols, x.data_ptr(), cols, res.data_ptr(), cols, fp.FT_BF16, w.data_ptr(), fp.FT_BF16, EPS, total.data_ptr(), cols,
                             y.data_ptr(), cols, q.data_ptr(), cols, scale.data_ptr(), groups, 0, stream())
    assert call(x, res, total, y) == 0
    assert y[1].isnan().all() and y[3, 0].isnan() and (y[3, 1:] == 0).all() and (y[4] == 0).all() and y[[0, 2, 5]].isfinite().all()
    assert scale[1].isnan().all() and scale[3, 0].isnan() and (scale[4] == 0).all() and (q[4] & 0x7F == 0).all()
    assert scale[[0, 2, 5]].isfinite().all()
    x2, res2 = x.clone(), res.clone()
    assert call(x2, res2, res2, x2) == 0   # the stream is updated in place, its norm replaces x
    assert torch.equal(bits(res2), bits(total)) and torch.equal(bits(x2), bits(y))
    x2, res2 = x.clone(), res.clone()
    assert call(x2, res2, x2, res2) == 0
    assert torch.equal(bits(x2), bits(total)) and torch.equal(bits(res2), bits(y))


@pytest.mark.parametrize("dtype", TYPES)
def test_rms_norm_8_bits_of_extreme_rows(pool, dtype):
    """Groups of tiny, huge and single values; only `sum`; no weight."""
    cols = 392
    x = torch.zeros(5, cols, device="cuda")
    x[0] = 1e-30
    x[1, 130] = 5.0
    x[2] = torch.arange(cols, device="cuda") - 200
    x[3] = 1e15
    x[4, :128] = 1e-12
    x[4, 128:] = 1.0
    x = x.to(dtype)
    groups = 4
    q, scale, y = torch.empty(5, cols, dtype=torch.uint8, device="cuda"), torch.empty(5, groups, device="cuda"), torch.empty_like(x)
    assert pool.rms_norm(5, cols, x.data_ptr(), cols, 0, 0, code(dtype), 0, fp.FT_F32, EPS, 0, 0, y.data_ptr(), cols, q.data_ptr(), cols, scale.data_ptr(), groups, 0,
                         stream()) == 0
    e6 = rms_formula(x, None, torch.ones(cols, device="cuda"))[2]
    wide = scale.double().repeat_interleave(128, 1)[:, :cols]
    within(q.view(torch.float8_e4m3fn).double() * wide, e6, 1.01 * E8 * e6.abs() + wide * 2.0 ** -10 * 1.01 + 60 * U * e6.abs(), "q")
    assert scale.isfinite().all() and scale[1, 0] == 0 and scale[1, 1] > 0
    total = torch.empty_like(x)
    assert pool.rms_norm(5, cols, x.data_ptr(), cols, x.data_ptr(), cols, code(dtype), 0, fp.FT_F32, EPS, total.data_ptr(), cols, 0, 0, stream=stream()) == 0
    assert torch.equal(total, x + x)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES + [(5000, 136), (2049, 77), (2600, 1000), (1400, 1784), (1400, 1592), (1300, 2040), (700, 2984), (660, 3848)])
def test_rms_norm_grad_against_64_bits(pool, shape, dtype, residual):
    rows, cols = shape
    g = gen(rows * 31 + cols)
    s = (randn(g, rows, cols) + 0.5).to(dtype)
    dy, w = randn(g, rows, cols).to(dtype), (1 + 0.1 * randn(g, cols)).to(torch.bfloat16)
    back = randn(g, rows, cols).to(dtype) if residual else None
    s6, r6, _ = rms_formula(s, None, w)
    rstd = r6[:, 0].float()
    ld = cols + 3 if cols % 2 else cols
    ss, gs, ds = strided(s, ld, 1 if cols % 2 else 0), strided(dy, ld + 8), strided(back, ld) if residual else None
    dx, dw = strided(torch.zeros_like(s), ld), torch.full((cols,), float("nan"), device="cuda")
    n = pool.rms_norm_grad_workspace(rows, cols)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")

    def call(out, dw, add):
        return pool.rms_norm_grad(rows, cols, gs.data_ptr(), ld + 8, ss.data_ptr(), ld, ds.data_ptr() if residual else 0, ld, code(dtype), w.data_ptr(),
                                  fp.FT_BF16, rstd.data_ptr(), out.data_ptr(), out.stride(0), dw.data_ptr() if dw is not None else 0, add, ws.data_ptr(), n, stream())

    assert call(dx, dw, False) == 0
    r6 = rstd.double()[:, None]
    xhat, a = s6 * r6, dy.double() * w.double()
    e6 = r6 * (a - xhat * (a * xhat).mean(1, keepdim=True))
    mag = r6 * (a.abs() + xhat.abs() * (a * xhat).abs().mean(1, keepdim=True))
    if residual:
        e6, mag = e6 + back.double(), mag + back.double().abs()
    within(dx, e6, 80 * U * mag + 1.01 * half_step(dtype) * e6.abs() + 1e-30, "dx")
    exp = (dy.double() * xhat).sum(0)
    within(dw, exp, (rows + 16) * U * (dy.double() * xhat).abs().sum(0) + 1e-30, "dweight")
    assert beside(dx).isnan().all() if ld > cols else True
    # the same bits again; accumulation adds once; dweight may be left out; dx may replace dy, and dsum
    dx2, dw2 = strided(torch.zeros_like(s), ld), dw.clone()
    assert call(dx2, dw2, True) == 0
    assert torch.equal(dw2, dw + dw) and torch.equal(bits(dx2), bits(dx))
    if residual:
        keep = ds.clone()
        assert call(ds, None, False) == 0
        assert torch.equal(bits(ds), bits(dx))
        ds.copy_(keep)
    assert call(gs, None, False) == 0
    assert torch.equal(bits(gs), bits(dx))


def test_rms_norm_grad_against_differences(pool):
    rows, cols = 5, 136
    g = gen(7)
    x, res, w, u, v = randn(g, rows, cols), randn(g, rows, cols), 1 + 0.1 * randn(g, cols), randn(g, rows, cols), randn(g, rows, cols)
    total, y, rstd, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty(cols, device="cuda")
    assert pool.rms_norm(rows, cols, x.data_ptr(), cols, res.data_ptr(), cols, fp.FT_F32, w.data_ptr(), fp.FT_F32, EPS, total.data_ptr(), cols,
                         y.data_ptr(), cols, rstd_ptr=rstd.data_ptr(), stream=stream()) == 0
    n = pool.rms_norm_grad_workspace(rows, cols)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    assert pool.rms_norm_grad(rows, cols, u.data_ptr(), cols, total.data_ptr(), cols, v.data_ptr(), cols, fp.FT_F32, w.data_ptr(), fp.FT_F32, rstd.data_ptr(),
                              dx.data_ptr(), cols, dw.data_ptr(), False, ws.data_ptr(), n, stream()) == 0

    def f(x, res, w):  # sum(u y) + sum(v s): dy = u, dsum = v
        s = x + res
        return (u.double() * s * (((s * s).mean(1, keepdim=True) + EPS) ** -0.5) * w).sum() + (v.double() * s).sum()

    at, h = [t.double() for t in (x, res, w)], 1e-5
    for k, grad in enumerate((dx, dx, dw)):
        d = torch.randn(at[k].shape, device="cuda", dtype=torch.float64, generator=g)
        up, down = ([t + s * d if i == k else t for i, t in enumerate(at)] for s in (h, -h))
        slope = (f(*up) - f(*down)) / (2 * h)
        # third derivatives are O(1) here: h^2 of them, and the products' roundings
        assert abs(float(slope - (grad.double() * d).sum())) <= 1e-5 * float((grad.double() * d).abs().sum()) + 1e-7


def test_rms_norm_refusals_and_empty_inputs(pool):
    x = torch.zeros(4, 256, device="cuda")
    w = torch.zeros(256, device="cuda")
    q, scale = torch.zeros(4, 256, dtype=torch.uint8, device="cuda"), torch.zeros(4, 2, device="cuda")
    X, W, Q, S = x.data_ptr(), w.data_ptr(), q.data_ptr(), scale.data_ptr()
    ok = dict(rows=4, cols=256, x_ptr=X, ldx=256, residual_ptr=X, ldr=256, dtype=fp.FT_F32, weight_ptr=W, param_dtype=fp.FT_F32, eps=EPS, sum_ptr=X, lds=256,
              y_ptr=X, ldy=256, q_ptr=Q, ldq=256, q_scale_ptr=S, ldqs=2)
    ok["sum_ptr"] = 0
    assert pool.rms_norm(**ok) == 0
    for bad in (dict(cols=0), dict(ldx=255), dict(ldr=255), dict(sum_ptr=X, lds=255), dict(ldy=255), dict(ldq=255), dict(ldqs=1), dict(dtype=2), dict(param_dtype=9),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x_ptr=0), dict(y_ptr=0, q_ptr=0, q_scale_ptr=0), dict(q_ptr=0),
                dict(q_scale_ptr=0), dict(x_ptr=X + 2), dict(residual_ptr=X + 1), dict(weight_ptr=W + 1), dict(q_scale_ptr=S + 2), dict(rstd_ptr=S + 1)):
        assert pool.rms_norm(**{**ok, **bad}) == INVALID, bad
    assert pool.rms_norm(**{**ok, "cols": (1 << 30) + 1, "ldx": 1 << 31, "ldy": 1 << 31}) == CAPACITY
    assert pool.rms_norm(**{**ok, "rows": 0, "x_ptr": 0, "y_ptr": 0}) == 0
    n = pool.rms_norm_grad_workspace(4, 256)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    dw = torch.full((256,), 3.0, device="cuda")
    ok = dict(rows=4, cols=256, dy_ptr=X, lddy=256, s_ptr=X, lds=256, dsum_ptr=X, lddsum=256, dtype=fp.FT_F32, weight_ptr=W, param_dtype=fp.FT_F32, rstd_ptr=W,
              dx_ptr=X, lddx=256, dweight_ptr=dw.data_ptr(), accumulate=False, ws_ptr=ws.data_ptr(), ws_bytes=n)
    for bad in (dict(cols=0), dict(lddy=1), dict(lds=1), dict(lddsum=1), dict(lddx=1), dict(dtype=7), dict(dy_ptr=0), dict(s_ptr=0), dict(dx_ptr=0), dict(rstd_ptr=0),
                dict(ws_ptr=0), dict(ws_ptr=ws.data_ptr() + 16), dict(dweight_ptr=dw.data_ptr() + 1), dict(dx_ptr=X + 1), dict(dsum_ptr=X + 2)):
        assert pool.rms_norm_grad(**{**ok, **bad}) == INVALID, bad
    assert pool.rms_norm_grad(**{**ok, "ws_bytes": n - 1}) == CAPACITY
    torch.cuda.synchronize()
    assert (dw == 3.0).all()
    assert pool.rms_norm_grad(**{**ok, "rows": 0, "accumulate": True, "ws_ptr": 0}) == 0 and (dw == 3.0).all()
    assert pool.rms_norm_grad(**{**ok, "rows": 0, "ws_ptr": 0}) == 0 and (dw == 0.0).all()


# ---- the gradients' norm ----------------------------------------------------------------------------------------

def grad_norm(pool, tensors, max_norm=1.0, more=None, want=True):
    n = pool.grad_norm_workspace()
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    total = torch.full((1,), float("nan"), dtype=torch.float64, device="cuda")
    norm, factor = torch.full((2, 1), float("nan"), device="cuda")
    listed = [fp.GradTensor(grad=t.data_ptr() if t.numel() else None, n=t.numel(), dtype=code(t.dtype)) for t in tensors]
    assert pool.grad_norm(listed, max_norm, 0 if more is None else more.data_ptr(), total.data_ptr(), norm.data_ptr() if want else 0,
                          factor.data_ptr() if want else 0, ws.data_ptr(), n, stream()) == 0
    return total, norm, factor


def check_norm(pool, tensors, max_norm=1.0):
    total, norm, factor = grad_norm(pool, tensors, max_norm)
    exp = sum(float(t.double().square().sum()) for t in tensors)
    # at most 32 squares are added in fp32, in two rows of 16; every square and every sum rounds
    assert abs(float(total) - exp) <= 20 * U * exp
    assert abs(float(norm) - math.sqrt(exp)) <= 12 * U * math.sqrt(exp)
    want = max_norm / math.sqrt(exp) if math.sqrt(exp) > max_norm else 1.0
    assert abs(float(factor) - want) <= 12 * U * want
    return total


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", [(1,), (7, 1), (4096,), (0, 5, 0, 4097), (16384, 3, 12345), (300001, 65536, 2), (1 << 22,)])
def test_grad_norm_against_64_bits(pool, sizes, dtype):
    g = gen(sum(sizes))
    flat = randn(g, sum(sizes) + 8).to(dtype)
    for shift in (0, 1, 3):  # tensors back to back, from any element on
        at, tensors = shift, []
        for n in sizes:
            tensors.append(flat[at:at + n])
            at += n
        first = check_norm(pool, tensors)
        assert torch.equal(first, check_norm(pool, tensors, 1e9))  # the same bits again


def test_grad_norm_of_many_tensors_of_both_types(pool):
    g = gen(2)
    tensors = [randn(g, 1 + 37 * i % 5000).to(TYPES[i % 2]) * 10.0 ** (i % 9 - 4) for i in range(1000)] + [randn(g, 3_000_000)]
    check_norm(pool, tensors)
    check_norm(pool, tensors[::-1])


def test_grad_norm_in_parts_and_over_ranks(pool):
    g = gen(4)
    parts = [randn(g, 50000 + i) for i in range(3)]
    whole, norm, factor = grad_norm(pool, parts, 2.5)
    sums = [grad_norm(pool, [t], want=False)[0] for t in parts]
    total, norm2, factor2 = grad_norm(pool, [], 2.5, more=sums[0] + sums[1] + sums[2])
    assert abs(float(total - whole)) <= 1e-15 * float(whole) and torch.equal(norm, norm2) and torch.equal(factor, factor2)
    chained = grad_norm(pool, parts[1:], 2.5, more=sums[0])
    assert abs(float(chained[0] - whole)) <= 40 * U * float(whole)
    n = pool.grad_norm_workspace()   # sumsq may be `more`
    ws, run = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    for t in parts:
        assert pool.grad_norm([fp.GradTensor(grad=t.data_ptr(), n=t.numel(), dtype=fp.FT_F32)], 0.0, run.data_ptr(), run.data_ptr(), 0, 0, ws.data_ptr(), n, stream()) == 0
    assert torch.equal(run, sums[0] + sums[1] + sums[2])


@pytest.mark.parametrize("dtype", TYPES)
def test_grad_norm_over_the_whole_range_and_of_bad_values(pool, dtype):
    g = gen(5)
    for scale in (1e-38, 1e-30, 1e-22, 1e-12, 1e18, 1e25, 1e36):
        check_norm(pool, [(randn(g, 5000).double() * scale).to(dtype)], scale)
    check_norm(pool, [torch.cat([torch.full((5000,), 1e-20, device="cuda"), torch.full((3,), 1e30, device="cuda")]).to(dtype)])
    total, norm, factor = grad_norm(pool, [torch.zeros(9999, dtype=dtype, device="cuda")])
    assert float(total) == 0 and float(norm) == 0 and float(factor) == 1
    assert [float(t) for t in grad_norm(pool, [], 0.5)] == [0.0, 0.0, 1.0]
    bad = randn(g, 70000).to(dtype)
    bad[69999] = float("inf")
    total, norm, factor = grad_norm(pool, [bad])
    assert float(norm) == math.inf and float(factor) == 0
    bad[5] = float("nan")
    assert all(t.isnan() for t in grad_norm(pool, [bad]))


def test_grad_norm_clips_an_adamw_step(pool):
    """The factor goes straight into pool_adamw_step: the same parameters as with gradients scaled beforehand (by one fp32 product)."""
    g = gen(6)
    grads = [randn(g, 5001), randn(g, 777)]
    n = pool.grad_norm_workspace()
    ws, factor = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(1, device="cuda")
    assert pool.grad_norm([fp.GradTensor(grad=t.data_ptr(), n=t.numel(), dtype=fp.FT_F32) for t in grads], 0.125, 0, 0, 0, factor.data_ptr(), ws.data_ptr(), n,
                          stream()) == 0
    assert 0 < float(factor) < 1

    def step(grads, scale):
        out = [(torch.ones_like(t), torch.zeros_like(t), torch.zeros_like(t)) for t in grads]
        tensors = [fp.AdamwTensor(param=p.data_ptr(), grad=t.data_ptr(), m=m.data_ptr(), v=v.data_ptr(), n=t.numel(), param_dtype=fp.FT_F32,
                                  grad_dtype=fp.FT_F32, state_bits=32) for t, (p, m, v) in zip(grads, out)]
        assert pool.adamw_step(tensors, fp.AdamwConfig(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=scale, step=1), stream()) == 0
        return out
    for a, b in zip(step(grads, factor.data_ptr()), step([t * factor for t in grads], None)):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_grad_norm_refusals(pool):
    t = torch.ones(64, device="cuda")
    n = pool.grad_norm_workspace()
    ws, d = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.zeros(2, dtype=torch.float64, device="cuda")
    W, D, T = ws.data_ptr(), d.data_ptr(), t.data_ptr()
    ok = dict(tensors=[fp.GradTensor(grad=T, n=64, dtype=fp.FT_F32)], max_norm=1.0, more_ptr=0, sumsq_ptr=D, norm_ptr=D + 8, factor_ptr=D + 12, ws_ptr=W, ws_bytes=n)

    def one(**change):
        return dict(tensors=[fp.GradTensor(**{**dict(grad=T, n=64, dtype=fp.FT_F32), **change})])
    assert pool.grad_norm(**ok) == 0
    for bad in (one(dtype=2), one(grad=None), one(grad=T + 2), dict(max_norm=-1.0), dict(max_norm=math.nan), dict(more_ptr=D + 4), dict(sumsq_ptr=D + 4),
                dict(norm_ptr=D + 1), dict(factor_ptr=D + 2), dict(ws_ptr=0), dict(ws_ptr=W + 8)):
        assert pool.grad_norm(**{**ok, **bad}) == INVALID, bad
    for bad in (one(n=(1 << 40) + 1), dict(ws_bytes=n - 1)):
        assert pool.grad_norm(**{**ok, **bad}) == CAPACITY, bad
    assert pool.grad_norm(**{**ok, **one(grad=None, n=0)}) == 0
    assert pool.grad_norm(**{**ok, "max_norm": math.nan, "factor_ptr": 0}) == 0
    assert pool.grad_norm(**{**ok, "max_norm": math.inf}) == 0


# ---- log probabilities ------------------------------------------------------------------------------------------

def score_inputs(seed, rows, hidden, vocab, valid, ldx=None, ldw=None):
    """x and w on grids on which every sum of products is exact in fp32: equal logits are equal whatever the order of the sums."""
    g = gen(seed)
    step = 2.0 ** math.ceil(math.log2(6 / math.sqrt(hidden) / 255))
    w = (torch.round(randn(g, vocab, hidden) * hidden ** -0.5 / step)).clamp_(-255, 255) * step
    tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    x = randn(g, rows, hidden) + 8 * torch.rand(rows, 1, device="cuda", generator=g) * w[tokens]
    x = (torch.round(x * 16) / 16).clamp_(-15, 15)
    tokens = torch.where(torch.rand(rows, device="cuda", generator=g) < valid, tokens, -100).int()
    return strided(x.bfloat16(), ldx or hidden), strided(w.bfloat16(), ldw or hidden), tokens


def in_order(z, top):
    """Ids of the `top` largest of each row, equal ones by ascending id."""
    return torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top]


def run_scores(pool, x, w, tokens, top=0, scale=1.0, ws_bytes=None, fill=0, entropy=True):
    rows, hidden = x.shape
    vocab = w.shape[0]
    out = dict(logprob=torch.full((rows,), float("nan"), device="cuda") if tokens is not None else None,
               entropy=torch.full((rows,), float("nan"), device="cuda") if entropy else None)
    if top:
        out.update(ids=torch.full((rows, top), -7, dtype=torch.int32, device="cuda"), top=torch.full((rows, top), float("nan"), device="cuda"))
    least, best = pool.token_logprobs_workspace(rows, hidden, vocab, top)
    n = best if ws_bytes is None else ws_bytes(least, best)
    ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
    at = {k: t.data_ptr() for k, t in out.items() if t is not None}
    rc = pool.token_logprobs(rows, hidden, vocab, x.data_ptr(), x.stride(0), w.data_ptr(), w.stride(0), 0 if tokens is None else tokens.data_ptr(), scale,
                             at.get("logprob", 0), at.get("entropy", 0), top, at.get("ids", 0), at.get("top", 0), ws.data_ptr(), n, stream())
    torch.cuda.synchronize()   # the workspace is freed with this call
    return rc, out


def check_scores(out, x, w, tokens, top, scale, exact_logits=True):
    rows, hidden = x.shape
    keep = torch.ones(rows, dtype=torch.bool, device="cuda") if tokens is None else tokens >= 0
    z = x[keep].double() @ w.double().T
    # a logit's error; the exponentials' 2 ulp of a product with the exponent, a sum over 4 terms a thread and 128 columns, then joins
    t_z = scale * (0 if exact_logits else 2 * U * (hidden + 8)) * (x[keep].double().abs() @ w.double().abs().T).amax(1)
    lse = torch.logsumexp(z * scale, 1)
    spread = (z.amax(1) - z.amin(1)) * scale
    t_lse = t_z + (64 + 0.02 * w.shape[0]) * U + 8 * U * (spread + lse.abs() + 16)
    logp = z * scale - lse[:, None]
    exp = -(logp.exp() * logp).sum(1)
    if out["entropy"] is not None:
        within(out["entropy"][keep], exp, (t_lse + 40 * U) * (1 + exp) * 2, "entropy")
        assert (out["entropy"][~keep] == 0).all()
    if tokens is not None:
        picked = logp.gather(1, tokens[keep].long()[:, None])[:, 0]
        within(out["logprob"][keep], picked, t_lse + t_z + 8 * U * picked.abs(), "logprob")
        assert (out["logprob"][~keep] == 0).all()
    if top:
        real = min(top, w.shape[0])
        ids = out["ids"][keep].long()
        best = in_order(z, real)
        if exact_logits:
            assert torch.equal(ids[:, :real], best)
        within(out["top"][keep][:, :real], logp.gather(1, best), (t_lse + t_z)[:, None] + 8 * U * logp.gather(1, best).abs(), "alternatives")
        assert (ids[:, real:] == -1).all() and (out["top"][keep][:, real:] == -math.inf).all()
        assert (out["ids"][~keep] == -1).all() and (out["top"][~keep] == 0).all()


SCORE_SHAPES = [(1, 8, 1, 1.0, 3), (1, 64, 257, 1.0, 32), (2, 8, 1000, 1.0, 1), (3, 72, 63, 1.0, 5), (64, 64, 256, 0.5, 8), (65, 136, 300, 0.7, 20), (127, 128, 511, 1.0, 4),
                (129, 256, 1025, 0.3, 32), (257, 520, 4099, 0.8, 8), (300, 1024, 2048, 0.01, 8), (513, 200, 777, 0.9, 7), (1000, 64, 5003, 0.5, 20), (24, 1032, 33000, 1.0, 8),
                (600, 4232, 3000, 0.9, 2), (40, 2048, 9001, 0.9, 16)]


@pytest.mark.parametrize("fill", [0, 255])
@pytest.mark.parametrize("shape", SCORE_SHAPES)
def test_logprobs_against_64_bits(pool, shape, fill):
    rows, hidden, vocab, valid, top = shape
    x, w, tokens = score_inputs(rows * 7 + vocab, rows, hidden, vocab, valid, hidden + 8, hidden + 16)
    for given, k, scale in ((tokens, top, 1.0), (tokens, 0, 1.0), (None, top, 0.7)):
        rc, out = run_scores(pool, x, w, given, k, scale, fill=fill)
        assert rc == 0
        check_scores(out, x, w, given, k, scale)
    rc, again = run_scores(pool, x, w, tokens, top, fill=255 - fill, entropy=False)
    assert rc == 0 and pool.status() == (0, 0)
    rc, first = run_scores(pool, x, w, tokens, top, fill=fill)
    for k in ("logprob", "ids", "top"):   # the same bits, whatever the workspace held
        assert torch.equal(bits(first[k]), bits(again[k]))


def test_logprobs_of_a_listed_token_is_its_place_in_the_list(pool):
    x, w, tokens = score_inputs(9, 300, 256, 3000, 0.9)
    rc, out = run_scores(pool, x, w, tokens, 8)
    hit = out["ids"] == tokens[:, None]
    assert rc == 0 and hit.any()
    assert torch.equal(out["top"][hit], out["logprob"][:, None].expand(-1, 8)[hit])


def test_logprobs_of_values_off_the_grid(pool):
    """Ordinary values: the logits are off by what the sums round; what is listed is as large as what should be."""
    g = gen(12)
    for rows, hidden, vocab in ((50, 4096, 5000), (700, 3584, 1500)):
        x, w = randn(g, rows, hidden).bfloat16(), (randn(g, vocab, hidden) * hidden ** -0.5).bfloat16()
        tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
        rc, out = run_scores(pool, x, w, tokens, 8)
        assert rc == 0
        check_scores(out, x, w, tokens, 8, 1.0, exact_logits=False)


@pytest.mark.parametrize("top", [1, 8, 32])
def test_logprobs_of_equal_logits(pool, top):
    """Ties go to the lowest id: all logits equal; a few values many times over; one that stands out; more places than tokens."""
    hidden, vocab = 64, 5000
    x = torch.zeros(5, hidden, device="cuda", dtype=torch.bfloat16)
    x[1:, 0] = 1
    x[2, 1] = 4
    x[3, 0] = -1
    x[4, 0] = -0.0
    w = torch.zeros(vocab, hidden, device="cuda", dtype=torch.bfloat16)
    w[:, 0] = (torch.arange(vocab, device="cuda") * 7 % 5).bfloat16()
    w[4321, 1] = 2
    tokens = torch.tensor([0, 1, 4321, 4999, 2], device="cuda", dtype=torch.int32)
    rc, out = run_scores(pool, x, w, tokens, top)
    assert rc == 0
    check_scores(out, x, w, tokens, top, 1.0)
    rc, out = run_scores(pool, x, w[:5], tokens % 5, top)
    assert rc == 0
    check_scores(out, x, w[:5], tokens % 5, top, 1.0)


def test_logprobs_of_extreme_logits(pool):
    """Infinities, NaN, far apart logits, and what they leave in the other rows."""
    hidden, vocab, top = 64, 700, 6
    x, w, _ = score_inputs(3, 7, hidden, vocab, 1.0)
    x, w = x.clone(), w.clone()
    w[:, 0], w[:, 1], w[:, 2] = 0, 0, 0
    w[5, 0], w[600, 0] = 1, -1
    w[:, 1] = 1
    x[:, :3] = 0
    x[1, 0] = 1e4           # one token certain: entropy 0, logprob 0
    x[2, 1] = 3e38          # all logits equally huge
    x[3, 0] = float("nan")
    x[4, 0] = float("inf")  # inf * 0: NaN everywhere, inf and -inf at two
    x[5] = 0                # all equal
    x[6, 0] = -2e4
    tokens = torch.tensor([3, 5, 9, 1, 2, 3, 600], device="cuda", dtype=torch.int32)
    rc, out = run_scores(pool, x, w, tokens, top)
    assert rc == 0
    for k in ("logprob", "entropy"):
        assert out[k][[3, 4]].isnan().all() and out[k][[0, 1, 2, 5, 6]].isfinite().all()
    assert out["top"][[3, 4]].isnan().all() and ((out["ids"] >= 0) & (out["ids"] < vocab)).all()
    assert out["logprob"][1] == 0 and out["entropy"][1] == 0 and out["ids"][1, 0] == 5 and out["ids"][6, 0] == 600
    keep = torch.tensor([0, 5], device="cuda")
    check_scores({k: v[keep] for k, v in out.items()}, x[keep], w, tokens[keep], top, 1.0)
    assert torch.equal(out["ids"][3], torch.arange(top, device="cuda", dtype=torch.int32)) and out["ids"][4, 0] == 5
    # logits of -inf: they count nothing and stand last
    w2, x2 = w.clone(), x[:1].clone()
    w2[:, 0] = 0
    w2[10:, 0] = float("-inf")
    x2[0, 0] = 1
    rc, out = run_scores(pool, x2, w2, tokens[:1], 12)
    assert rc == 0
    z = (x2[0, 1:].double() @ w2[:10, 1:].double().T)
    assert out["ids"][0].tolist() == z.sort(descending=True, stable=True).indices.tolist() + [10, 11]
    within(out["top"][0, :10], torch.log_softmax(z, 0).sort(descending=True).values, 1e-5, "finite ones")
    assert (out["top"][0, 10:] == -math.inf).all() and out["logprob"].isfinite().all() and out["entropy"].isfinite().all()


@pytest.mark.parametrize("top", [0, 5])
def test_logprobs_in_pieces(pool, top):
    """Any workspace between the least and the best gives the same bits."""
    x, w, tokens = score_inputs(5, 1300, 72, 1111, 0.6)
    tokens[256:512] = -100  # a piece in which nothing counts
    least, best = pool.token_logprobs_workspace(1300, 72, 1111, top)
    assert least < best
    for given in (tokens, None):
        rc, first = run_scores(pool, x, w, given, top)
        assert rc == 0
        check_scores(first, x, w, given, top, 1.0)
        for n in (least, (least + best) // 2, best + 4096):
            rc, out = run_scores(pool, x, w, given, top, ws_bytes=lambda *_: n, fill=255)
            assert rc == 0
            assert all(torch.equal(bits(out[k]), bits(first[k])) for k in out if out[k] is not None)


def test_logprobs_bad_tokens_are_reported_and_skipped(pool):
    x, w, tokens = score_inputs(8, 90, 64, 500, 0.8)
    tokens[7], tokens[30], tokens[80] = 500, -1, -100
    x[7], x[80] = float("nan"), float("inf")
    rc, out = run_scores(pool, x, w, tokens, 4)
    assert rc == 0
    assert pool.status() == (BAD_ID, 7)
    masked = torch.where((tokens >= 0) & (tokens < 500), tokens, -100)
    check_scores(out, x, w, masked, 4, 1.0)
    assert pool.status() == (0, 0)
    rc, out = run_scores(pool, x, w, torch.full_like(tokens, -100), 4)   # nothing counts
    assert rc == 0 and (out["logprob"] == 0).all() and (out["entropy"] == 0).all() and (out["ids"] == -1).all()


def test_logprobs_refusals_and_empty_inputs(pool):
    rows, hidden, vocab, top = 4, 16, 32, 3
    x, w = torch.zeros(rows, hidden, device="cuda").bfloat16(), torch.zeros(vocab, hidden, device="cuda").bfloat16()
    f, i = torch.full((64,), 3.0, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    least, _ = pool.token_logprobs_workspace(rows, hidden, vocab, top)
    ws = torch.zeros(least, dtype=torch.uint8, device="cuda")
    X, W, F, I, S = x.data_ptr(), w.data_ptr(), f.data_ptr(), i.data_ptr(), ws.data_ptr()
    ok = dict(rows=rows, hidden=hidden, vocab=vocab, x_ptr=X, ldx=hidden, w_ptr=W, ldw=hidden, tokens_ptr=I, logit_scale=1.0, logprob_ptr=F, entropy_ptr=F + 64,
              top=top, top_ids_ptr=I + 64, top_logprobs_ptr=F + 128, ws_ptr=S, ws_bytes=least)
    assert pool.token_logprobs(**ok) == 0
    torch.cuda.synchronize()
    f.fill_(3.0)
    for bad in (dict(hidden=0), dict(hidden=12), dict(vocab=0), dict(x_ptr=0), dict(x_ptr=X + 8), dict(ldx=8), dict(ldx=20), dict(w_ptr=0), dict(w_ptr=W + 2), dict(ldw=8),
                dict(tokens_ptr=0), dict(logprob_ptr=0), dict(tokens_ptr=I + 1), dict(logit_scale=0.0), dict(logit_scale=-1.0), dict(logit_scale=math.nan),
                dict(logit_scale=math.inf), dict(logprob_ptr=F + 2), dict(entropy_ptr=F + 1), dict(top_ids_ptr=0), dict(top_logprobs_ptr=0), dict(top_ids_ptr=I + 2),
                dict(ws_ptr=0), dict(ws_ptr=S + 128)):
        assert pool.token_logprobs(**{**ok, **bad}) == INVALID, bad
    for bad in (dict(top=33), dict(ws_bytes=least - 1), dict(rows=1 << 31), dict(vocab=1 << 31)):
        assert pool.token_logprobs(**{**ok, **bad}) == CAPACITY, bad
    torch.cuda.synchronize()
    assert (f == 3.0).all()
    assert pool.token_logprobs(**{**ok, "rows": 0, "ws_ptr": 0}) == 0
    with pytest.raises(fp.FlowpoolError):
        pool.token_logprobs_workspace(rows, 12, vocab, top)
    with pytest.raises(fp.FlowpoolError):
        pool.token_logprobs_workspace(rows, hidden, vocab, 33)


@pytest.mark.parametrize("rows", [20, 60, 100, 200, 600])
def test_a_logprobs_wait_that_runs_out_reports_timeout_and_leaves_the_context_usable(rows):
    """Under the test hook every load announces 16 bytes more than it brings, so no stage is ever seen complete although all
    arrive: every warp of every pair waits a millisecond, gives up, waits once more for what it has under way, and returns."""
    p = new_pool()
    x, w, tokens = score_inputs(rows, rows, 136, 1000, 0.9)
    rc, first = run_scores(p, x, w, tokens, 4)
    assert rc == 0 and p.status() == (0, 0)
    assert p.set_tuning(bulk_timeout_test=1, bulk_wait_limit_us=1000) == 0
    assert run_scores(p, x, w, tokens, 4)[0] == 0
    code, detail = p.status()
    assert code == TIMEOUT and detail < torch.cuda.get_device_properties(0).multi_processor_count
    assert p.set_tuning() == 0
    rc, again = run_scores(p, x, w, tokens, 4)
    assert rc == 0 and p.status() == (0, 0)
    for k in first:
        assert torch.equal(bits(first[k]), bits(again[k]))
    p.destroy()


# ---- together ---------------------------------------------------------------------------------------------------

def test_the_operators_on_another_stream_and_in_a_graph(pool):
    rows, cols, vocab, heads, dim = 200, 256, 1500, 4, 64
    x, w, tokens = score_inputs(21, rows, cols, vocab, 0.8)
    g = gen(22)
    res, weight, dy = randn(g, rows, cols).bfloat16(), 1 + 0.1 * randn(g, cols), randn(g, rows, cols).bfloat16()
    pos = torch.randint(0, 1000, (3, rows), device="cuda", generator=g, dtype=torch.int32)
    cfg = fp.rotary_config(1e4 ** (-np.arange(32) / 32), np.arange(32) % 3, dim)
    out = dict(turned=torch.empty(rows, heads * dim, device="cuda").bfloat16(), total=torch.empty_like(res), y=torch.empty_like(res), rstd=torch.empty(rows, device="cuda"),
               dx=torch.empty_like(res), dw=torch.empty(cols, device="cuda"), norm=torch.empty(1, device="cuda"), factor=torch.empty(1, device="cuda"),
               logprob=torch.empty(rows, device="cuda"), entropy=torch.empty(rows, device="cuda"), ids=torch.empty(rows, 4, dtype=torch.int32, device="cuda"),
               top=torch.empty(rows, 4, device="cuda"))
    sizes = pool.rms_norm_grad_workspace(rows, cols), pool.grad_norm_workspace(), pool.token_logprobs_workspace(rows, cols, vocab, 4)[1]
    ws = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes]
    o = {k: t.data_ptr() for k, t in out.items()}
    turn = [fp.RotaryTensor(src=x.data_ptr(), dst=o["turned"], src_row=cols, src_head=dim, dst_row=cols, dst_head=dim, heads=heads, dtype=fp.FT_BF16)]
    grads = [fp.GradTensor(grad=o["dw"], n=cols, dtype=fp.FT_F32), fp.GradTensor(grad=o["dx"], n=rows * cols, dtype=fp.FT_BF16)]

    def step(st):
        assert pool.rotary(rows, pos.data_ptr(), rows, cfg, turn, st) == 0
        assert pool.rms_norm(rows, cols, o["turned"], cols, res.data_ptr(), cols, fp.FT_BF16, weight.data_ptr(), fp.FT_F32, EPS, o["total"], cols, o["y"], cols,
                             rstd_ptr=o["rstd"], stream=st) == 0
        assert pool.token_logprobs(rows, cols, vocab, o["y"], cols, w.data_ptr(), cols, tokens.data_ptr(), 1.0, o["logprob"], o["entropy"], 4, o["ids"], o["top"],
                                   ws[2].data_ptr(), sizes[2], st) == 0
        assert pool.rms_norm_grad(rows, cols, dy.data_ptr(), cols, o["total"], cols, o["y"], cols, fp.FT_BF16, weight.data_ptr(), fp.FT_F32, o["rstd"], o["dx"], cols,
                                  o["dw"], False, ws[0].data_ptr(), sizes[0], st) == 0
        assert pool.grad_norm(grads, 1.0, 0, 0, o["norm"], o["factor"], ws[1].data_ptr(), sizes[1], st) == 0

    step(stream())
    torch.cuda.synchronize()
    first = {k: t.clone() for k, t in out.items()}
    exp = math.sqrt(float(out["dw"].double().square().sum() + out["dx"].double().square().sum()))
    assert abs(float(out["norm"]) - exp) <= 12 * U * exp

    def same():
        torch.cuda.synchronize()
        for k, t in out.items():
            assert torch.equal(bits(t), bits(first[k])), k
            t.zero_()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(side.cuda_stream)
    same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream().cuda_stream)
    for _ in range(2):
        graph.replay()
        same()
