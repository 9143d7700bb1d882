"""The operators of the backbone's last layer and of its optimizer, as measurable cases.

A training step over an assembled microbatch ends with a layer norm, the token loss over the vocabulary, their
gradients, and an optimizer step over the embedding table and the other weights.  Every case below is one pass through
one of these operators, either in a plain form (elementary torch operations in 32 bits) or, where `own` is set, through
the library's own calls.

  norm       y = (x - mean) * rstd * weight + bias, with the row statistics
  norm_grad  its gradients towards x, weight and bias
  loss       per-row -log softmax(x W^T)[label] and log-sum-exp; rows labelled -100 count nothing
  loss_grad  the same together with its gradients towards x and W
  adamw      one AdamW step over many tensors, states held in 32 or in 8 bits
"""
import math

import torch

own = False

IGNORE = -100
EPS = 1e-5
BLOCK = 256          # elements that share one scale in 8-bit states
FP8_MAX = 448.0      # largest value of float8_e4m3fn
FP8_TINY = 2.0 ** -9  # its smallest positive value
LR, BETA1, BETA2, ADAM_EPS, DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1


def listed():
    return [
        # one token of a sequence that is being written: latency alone
        dict(name="norm_one_row", op="norm", rows=1, cols=3584, dtype="bfloat16"),
        # a packed microbatch at its full token budget
        dict(name="norm_microbatch", op="norm", rows=32768, cols=3584, dtype="bfloat16"),
        # an odd packed batch of odd width kept in 32 bits (an encoder's output before the cast on write)
        dict(name="norm_grad_ragged", op="norm_grad", rows=4099, cols=1023, dtype="float32"),
        # the backward pass of a full microbatch
        dict(name="norm_grad_microbatch", op="norm_grad", rows=32768, cols=3584, dtype="bfloat16"),
        # scoring a few rows: the weights are read once, nothing else counts
        dict(name="loss_few_rows", op="loss", rows=24, hidden=1024, vocab=32768, valid=1.0),
        # evaluation of a microbatch whose image placeholders (a third here) have no label
        dict(name="loss_microbatch", op="loss", rows=16384, hidden=3584, vocab=32768, valid=0.66),
        # a microbatch of the smallest configuration: budget 4096, hidden 1024
        dict(name="loss_grad_small", op="loss_grad", rows=4096, hidden=1024, vocab=32768, valid=0.6),
        # odd sizes everywhere: the tail of a batch against a vocabulary that no tile divides
        dict(name="loss_grad_ragged", op="loss_grad", rows=1777, hidden=4104, vocab=50021, valid=0.9),
        # a microbatch of the image mix at its full budget, text and image tokens half and half
        dict(name="loss_grad_microbatch", op="loss_grad", rows=32768, hidden=3584, vocab=32768, valid=0.5),
        # the weights and biases of two norms: latency alone
        dict(name="adamw_norm_weights", op="adamw", sizes="3584,3584,3584,3584", param="float32", grad="float32", bits=32,
             copy=False, align=128),
        # the embedding table and its norm: 32-bit master weights, the 16-bit table that assembly reads written beside them
        dict(name="adamw_table", op="adamw", sizes="117440512,3584,3584", param="float32", grad="float32", bits=32,
             copy=True, align=128),
        # a block's projections and odd-sized extras in 16 bits, 8-bit states, tensors back to back in one buffer
        dict(name="adamw_8bit_ragged", op="adamw", sizes="12845056,12845056,1835008,1835008,52428800,3584,3584,1001,17",
             param="bfloat16", grad="bfloat16", bits=8, copy=False, align=1),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _width(rng, low):
    """A width that a 16-byte access divides (8 elements of 16 bits), none of the round ones."""
    c = 8 * _log_int(rng, low, 1024)
    return c + 8 if c % 1024 == 0 else c


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "loss", "loss_grad", "loss_grad", "adamw"])
    if op in ("norm", "norm_grad"):
        cols = rng.choice([1024, 3584, 4096, 8192, _log_int(rng, 40, 8191) | 1, _width(rng, 8)])
        rows = min(_log_int(rng, 1, 131072), 32768 * 3584 // cols)
        return dict(op=op, rows=rows, cols=cols, dtype=rng.choice(["bfloat16", "bfloat16", "float32"]))
    if op in ("loss", "loss_grad"):
        hidden = rng.choice([1024, 3584, 4096, _width(rng, 16)])
        vocab = rng.choice([32768, _log_int(rng, 1000, 131072)])
        rows = min(_log_int(rng, 1, 32768), 16384 * 32768 * 3584 // (vocab * hidden), (1 << 30) // vocab)
        return dict(op=op, rows=rows, hidden=hidden, vocab=vocab, valid=rng.choice([1.0, round(rng.uniform(0.2, 1.0), 3)]))
    total, sizes = _log_int(rng, 1000, 100_000_000), []
    for _ in range(rng.randint(1, 24)):
        sizes.append(max(1, int(total * rng.uniform(0.01, 0.3))))
        total -= sizes[-1]
        if total < 1:
            break
    param = rng.choice(["float32", "bfloat16"])
    return dict(op="adamw", sizes=",".join(map(str, sizes)), param=param, grad=rng.choice(["float32", "bfloat16"]),
                bits=rng.choice([8, 32]), copy=param == "float32" and rng.random() < 0.5, align=rng.choice([1, 128, 128]))


# ---- inputs -----------------------------------------------------------------------------------------------------

def _sizes(case):
    """(sizes, element offset of each tensor in the flat buffers, buffer length, block offset, blocks in all)"""
    sizes = [int(s) for s in case["sizes"].split(",")]
    offs, blocks, at, b = [], [], 0, 0
    for n in sizes:
        offs.append(at)
        blocks.append(b)
        at += -(-n // case["align"]) * case["align"]
        b += -(-n // BLOCK)
    return sizes, offs, at, blocks, b


def _valid_rows(case):
    return max(1, round(case["rows"] * case["valid"]))


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    op = case["op"]
    s = {"case": case}
    if op in ("norm", "norm_grad"):
        r, c, t = case["rows"], case["cols"], getattr(torch, case["dtype"])
        # a residual stream: a few columns far larger than the rest, rows of differing scale and mean
        x = normal(r, c) * torch.exp(0.5 * normal(r, 1)) * torch.where(torch.rand(c, device="cuda", generator=g) < 0.01, 8.0, 1.0)
        s["x"] = (x + 0.3 * normal(r, 1)).to(t)
        s["weight"], s["bias"] = 1 + 0.1 * normal(c), 0.1 * normal(c)
        if op == "norm_grad":
            x = s["x"].double()
            mean = x.mean(1)
            s["mean"] = mean.float()
            s["rstd"] = ((x - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
            s["dy"] = (1e-2 * normal(r, c)).to(t)
    elif op in ("loss", "loss_grad"):
        r, h, v = case["rows"], case["hidden"], case["vocab"]
        w = (normal(v, h) * (1.2 / math.sqrt(h))).to(torch.bfloat16)
        u = torch.rand(r, device="cuda", generator=g)
        labels = (torch.exp(u * math.log(v)) - 1).long().clamp_(0, v - 1)  # token ids with a Zipf-like head
        # the model is sure of some targets and has no idea of others
        x = normal(r, h) + torch.rand(r, 1, device="cuda", generator=g) * 10 * w[labels].float()
        keep = torch.rand(r, device="cuda", generator=g).argsort() < _valid_rows(case)
        s.update(x=x.to(torch.bfloat16), w=w, labels=torch.where(keep, labels, IGNORE).to(torch.int32))
        if op == "loss_grad":
            s["grad_loss"] = torch.full((1,), 1.0 / _valid_rows(case), device="cuda")  # the mean over the rows that count
    else:
        sizes, offs, n, blocks, nb = _sizes(case)
        s["step"] = 100
        p = 0.02 * normal(n)
        s["param"] = p.to(getattr(torch, case["param"]))
        if case["copy"]:
            s["copy"] = p.to(torch.bfloat16)
        del p
        scale = torch.exp(1.5 * normal(n))  # elements of one tensor see gradients of very different size
        s["grad"] = (1e-3 * scale * normal(n)).to(getattr(torch, case["grad"]))
        m, r = 3e-4 * scale * normal(n), 1e-3 * scale * (0.5 + torch.rand(n, device="cuda", generator=g))
        if case["bits"] == 32:
            s["m"], s["v"] = m, r.square()
        else:
            for key, val, floor in (("m", m, False), ("r", r, True)):
                q, f = torch.zeros(n, device="cuda", dtype=torch.float8_e4m3fn), torch.zeros(nb, device="cuda")
                for size, o, b in zip(sizes, offs, blocks):
                    q[o:o + size], f[b:b - (-size // BLOCK)] = _pack8(val[o:o + size], floor)
                s[key], s[key + "_scale"] = q, f
    return s


_library = {}


def _pool():
    """The library's handle, made once for the process (its pages serve nothing here)."""
    if not _library:
        from paper_2606_23087_b200 import binding
        pool = binding.Pool(binding.PoolConfig(page_bytes=4096, hbm_pages=1, max_text_tokens=1024, hidden=8, max_samples=1,
                                               max_spans_per_sample=1, max_pages_per_span=1, max_seq_len=1))
        if pool.rc:
            raise binding.FlowpoolError(pool.rc, "pool_create")
        _library.update(pool=pool, binding=binding)
    return _library["pool"], _library["binding"]


def prepare(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    # output buffers, and with the library its handle, workspace and tensor list: a training program keeps them from step to step
    if op == "norm":
        s["y"] = torch.empty_like(s["x"])
        s["mean"], s["rstd"] = torch.empty(2, case["rows"], device="cuda")
    elif op == "norm_grad":
        s["dx"] = torch.empty_like(s["x"])
        s["dweight"], s["dbias"] = torch.empty(2, case["cols"], device="cuda")
    elif op in ("loss", "loss_grad"):
        s["loss"], s["lse"] = torch.empty(2, case["rows"], device="cuda")
        if op == "loss_grad":
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
    if own:
        pool, fp = _pool()
        s["pool"], s["fp"] = pool, fp
        if op == "norm_grad":
            s["ws_bytes"] = pool.layer_norm_grad_workspace(case["rows"], case["cols"])
        elif op in ("loss", "loss_grad"):
            s["ws_bytes"] = pool.token_loss_workspace(case["rows"], case["hidden"], case["vocab"], op == "loss_grad", fp.FT_BF16)[1]
        elif op == "adamw":
            sizes, offs, _, blocks, _ = _sizes(case)
            code = {"float32": fp.FT_F32, "bfloat16": fp.FT_BF16}

            def at(key, o):
                return s[key].data_ptr() + o * s[key].element_size() if key in s else None

            second = "v" if case["bits"] == 32 else "r"
            s["tensors"] = (fp.AdamwTensor * len(sizes))(*[
                fp.AdamwTensor(param=at("param", o), grad=at("grad", o), m=at("m", o), v=at(second, o), m_scale=at("m_scale", b),
                               v_scale=at("r_scale", b), copy=at("copy", o), n=n, weight_decay=DECAY,
                               param_dtype=code[case["param"]], grad_dtype=code[case["grad"]], state_bits=case["bits"])
                for n, o, b in zip(sizes, offs, blocks)])
        if s.get("ws_bytes"):
            s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------

def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    y = d * rstd * s["weight"] + s["bias"]
    return {"y": y.to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}


def _plain_norm_grad(s):
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xhat = (s["x"].float() - s["mean"][:, None]) * rstd
    wdy = dy * s["weight"]
    dx = rstd * (wdy - wdy.mean(1, keepdim=True) - xhat * (wdy * xhat).mean(1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xhat).sum(0), "dbias": dy.sum(0)}


def _plain_loss(s, grad):
    valid = s["labels"] >= 0
    target = torch.where(valid, s["labels"], 0).long()[:, None]
    x = torch.where(valid[:, None], s["x"].float(), 0.0)
    w = s["w"].float()
    logits = x @ w.T
    top = logits.max(1, keepdim=True).values
    picked = logits.gather(1, target)
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    lse = torch.log(total) + top
    out = {"loss": torch.where(valid, (lse - picked)[:, 0], 0.0), "lse": torch.where(valid, lse[:, 0], 0.0)}
    if grad:
        del logits
        d = e.div_(total)
        d.scatter_add_(1, target, torch.full_like(picked, -1.0))
        d.mul_(torch.where(valid, s["grad_loss"], 0.0)[:, None])
        out.update(dx=(d @ w).to(s["x"].dtype), dw=(d.T @ x).to(s["w"].dtype))
    return out


def _pack8(val, floor):
    """A tensor in blocks of 256 as float8 values and one power-of-two scale a block; `floor`: what is positive stays positive."""
    n = val.numel()
    b = torch.nn.functional.pad(val, (0, -n % BLOCK)).view(-1, BLOCK)
    top = b.abs().amax(1)
    # the smallest power of two that brings the largest value to 448 or less
    mant, ex = torch.frexp(top)
    ex = (ex - 9 + (mant > FP8_MAX / 512).to(ex.dtype)).clamp_(-100, 100)
    scale = torch.where(top > 0, torch.ldexp(torch.ones_like(top), ex), 0.0)
    inv = torch.where(top > 0, torch.ldexp(torch.ones_like(top), -ex), 0.0)
    q = b * inv[:, None]
    if floor:
        q = torch.where((q > 0) & (q < FP8_TINY), FP8_TINY, q)
    return q.reshape(-1)[:n].to(torch.float8_e4m3fn), scale


def _unpack8(q, scale):
    n = q.numel()
    return q.float() * scale[:, None].expand(-1, BLOCK).reshape(-1)[:n]


def _plain_adamw_one(s, case, n, o, b):
    p, g = s["param"][o:o + n], s["grad"][o:o + n].float()
    bits8, nb = case["bits"] == 8, -(-n // BLOCK)
    if bits8:
        m = _unpack8(s["m"][o:o + n], s["m_scale"][b:b + nb])
        r = _unpack8(s["r"][o:o + n], s["r_scale"][b:b + nb])
        v = r * r
    else:
        m, v = s["m"][o:o + n], s["v"][o:o + n]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * (g * g)
    r = torch.sqrt(v)
    c1, c2 = 1 - BETA1 ** s["step"], math.sqrt(1 - BETA2 ** s["step"])
    new = p.float() * (1 - LR * DECAY) - (LR / c1) * m / (r * (1 / c2) + ADAM_EPS)
    p.copy_(new)
    if case["copy"]:
        s["copy"][o:o + n] = new.to(torch.bfloat16)
    if bits8:
        s["m"][o:o + n], s["m_scale"][b:b + nb] = _pack8(m, False)
        s["r"][o:o + n], s["r_scale"][b:b + nb] = _pack8(r, True)
    else:
        s["m"][o:o + n], s["v"][o:o + n] = m, v


_STATE = ("param", "copy", "m", "v", "r", "m_scale", "r_scale")


def _plain_adamw(s):
    case = s["case"]
    s["step"] += 1
    sizes, offs, _, blocks, _ = _sizes(case)
    [_plain_adamw_one(s, case, n, o, b) for n, o, b in zip(sizes, offs, blocks)]
    return {k: s[k] for k in _STATE if k in s}


# ---- the library's calls ----------------------------------------------------------------------------------------

def _own(s):
    case, pool, fp = s["case"], s["pool"], s["fp"]
    op, st = case["op"], torch.cuda.current_stream().cuda_stream
    p = {k: t.data_ptr() for k, t in s.items() if isinstance(t, torch.Tensor)}
    if op == "norm":
        code = fp.FT_BF16 if case["dtype"] == "bfloat16" else fp.FT_F32
        rc = pool.layer_norm(case["rows"], case["cols"], p["x"], case["cols"], code, p["weight"], p["bias"], fp.FT_F32, EPS,
                             p["y"], case["cols"], p["mean"], p["rstd"], st)
        out = ("y", "mean", "rstd")
    elif op == "norm_grad":
        code, c = fp.FT_BF16 if case["dtype"] == "bfloat16" else fp.FT_F32, case["cols"]
        rc = pool.layer_norm_grad(case["rows"], c, p["dy"], c, p["x"], c, code, p["weight"], fp.FT_F32, p["mean"], p["rstd"],
                                  p["dx"], c, p["dweight"], p["dbias"], False, p["ws"], s["ws_bytes"], st)
        out = ("dx", "dweight", "dbias")
    elif op == "loss":
        h = case["hidden"]
        rc = pool.token_loss(case["rows"], h, case["vocab"], p["x"], h, p["w"], h, p["labels"], p["loss"], p["lse"],
                             p["ws"], s["ws_bytes"], st)
        out = ("loss", "lse")
    elif op == "loss_grad":
        h = case["hidden"]
        rc = pool.token_loss_grad(case["rows"], h, case["vocab"], p["x"], h, p["w"], h, p["labels"], p["grad_loss"], 0,
                                  p["loss"], p["lse"], p["dx"], h, p["dw"], fp.FT_BF16, False, p["ws"], s["ws_bytes"], st)
        out = ("loss", "lse", "dx", "dw")
    else:
        s["step"] += 1
        cfg = fp.AdamwConfig(lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, step=s["step"])
        rc = pool.adamw_step(s["tensors"], cfg, st)
        out = [k for k in _STATE if k in s]
    if rc:
        raise fp.FlowpoolError(rc, op)
    return {k: s[k] for k in out}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "norm":
        return _plain_norm(state)
    if op == "norm_grad":
        return _plain_norm_grad(state)
    if op == "adamw":
        return _plain_adamw(state)
    return _plain_loss(state, op == "loss_grad")


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op in ("norm", "norm_grad"):
        r, c, e = case["rows"], case["cols"], 2 if case["dtype"] == "bfloat16" else 4
        if op == "norm":
            return {"bytes": 2 * r * c * e + 8 * c + 8 * r, "flops": 8 * r * c}
        return {"bytes": 3 * r * c * e + 12 * c + 8 * r, "flops": 14 * r * c}
    if op in ("loss", "loss_grad"):
        n, r, h, v = _valid_rows(case), case["rows"], case["hidden"], case["vocab"]
        if op == "loss":
            return {"bytes": 2 * n * h + 2 * v * h + 12 * r, "flops": 2 * n * h * v}
        return {"bytes": 2 * n * h + 2 * r * h + 4 * v * h + 12 * r, "flops": 6 * n * h * v}
    n = sum(_sizes(case)[0])
    each = 2 * (4 if case["param"] == "float32" else 2) + (4 if case["grad"] == "float32" else 2) + (2 if case["copy"] else 0)
    each += 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": each * n, "flops": 16 * n}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    d = {k: t.double() for k, t in s.items() if isinstance(t, torch.Tensor) and t.is_floating_point()}
    op = case["op"]
    if op == "norm":
        var, mean = torch.var_mean(d["x"], dim=1, unbiased=False)
        rstd = (var + EPS) ** -0.5
        return {"y": torch.addcmul(d["bias"], (d["x"] - mean[:, None]) * rstd[:, None], d["weight"]), "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        # dx = J^T (w dy), J = rstd (I - 1/c - xhat xhat^T / c), written out with the row's two projections
        a = d["dy"] * d["weight"]
        xhat = (d["x"] - d["mean"][:, None]) * d["rstd"][:, None]
        along = torch.einsum("rc,rc->r", a, xhat) / case["cols"]
        dx = (a - (a.sum(1) / case["cols"])[:, None] - along[:, None] * xhat) * d["rstd"][:, None]
        return {"dx": dx, "dweight": torch.einsum("rc,rc->c", d["dy"], xhat), "dbias": torch.einsum("rc->c", d["dy"])}
    if op in ("loss", "loss_grad"):
        r, h, v = case["rows"], case["hidden"], case["vocab"]
        rows = torch.nonzero(s["labels"] != IGNORE)[:, 0]
        y = s["labels"][rows].long()
        x = d["x"][rows]
        z = torch.mm(x, d["w"].T)
        lse = torch.logsumexp(z, 1)
        zero = torch.zeros(r, dtype=torch.float64, device="cuda")
        out = {"loss": zero.index_copy(0, rows, lse - z[torch.arange(len(y), device="cuda"), y]), "lse": zero.index_copy(0, rows, lse)}
        if op == "loss_grad":
            z.sub_(lse[:, None]).exp_()
            z[torch.arange(len(y), device="cuda"), y] -= 1
            z *= d["grad_loss"]
            dx = torch.zeros(r, h, dtype=torch.float64, device="cuda")
            dx[rows] = torch.mm(z, d["w"])
            out.update(dx=dx, dw=torch.mm(z.T, x))
        return out
    sizes, offs, _, blocks, nb = _sizes(case)
    t = s["step"] + 1
    out = {k: d[k].clone() for k in _STATE if k in d}
    for n, o, b in zip(sizes, offs, blocks):
        e, nblk = slice(o, o + n), -(-n // BLOCK)
        owner = torch.arange(n, device="cuda") // BLOCK + b
        if case["bits"] == 8:
            m0, v0 = d["m"][e] * d["m_scale"][owner], (d["r"][e] * d["r_scale"][owner]) ** 2
        else:
            m0, v0 = d["m"][e], d["v"][e]
        m = m0 + (1 - BETA1) * (d["grad"][e] - m0)
        v = v0 + (1 - BETA2) * (d["grad"][e] ** 2 - v0)
        step = (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + ADAM_EPS)
        out["param"][e] = d["param"][e] - LR * (DECAY * d["param"][e] + step)
        if case["copy"]:
            out["copy"][e] = out["param"][e]
        if case["bits"] == 32:
            out["m"][e], out["v"][e] = m, v
            continue
        for key, val in (("m", m), ("r", v ** 0.5)):
            top = torch.zeros(nblk, dtype=torch.float64, device="cuda").scatter_reduce_(0, owner - b, val.abs(), "amax")
            scale = torch.where(top > 0, 2.0 ** torch.ceil(torch.log2(top / FP8_MAX)).clamp(-100, 100), 0.0)
            q = torch.where(top[owner - b] > 0, val / scale[owner - b], 0.0)
            # the nearest value of the format: 3 bits behind the leading one, multiples of 2^-9 below 2^-6
            unit = 2.0 ** (torch.floor(torch.log2(q.abs().clamp_min(2.0 ** -6))) - 3)
            q = torch.round(q / unit) * unit
            out[key][e] = torch.where((val > 0) & (q == 0), FP8_TINY, q) if key == "r" else q
            out[key + "_scale"][b:b + nblk] = scale
    return out
