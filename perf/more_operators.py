"""Operators between an assembled microbatch and the optimizer, as measurable cases.

Every case is one pass through one operator, either in a plain form (elementary torch operations in 32 bits, 64 where those
lose what matters) or, where `own` is set, through the library's own calls.

  rotary    rotary positions with several axes over the heads of queries and keys; backward the same with the angle negated
  rms       s = x + residual, y = s / sqrt(mean(s^2) + eps) * weight, in 16 or 32 bits or as float8 with a scale per 128 columns
  rms_grad  its gradients towards s (which are x's and the residual's) and weight
  grad_norm the 2-norm over many gradients, and the factor that brings it down to a limit
  logprobs  log softmax(x W^T) at given tokens, the entropy, and the likeliest alternatives
"""
import math

import torch

own = False

IGNORE = -100
EPS = 1e-6
GROUP = 128      # columns that share a scale in 8-bit outputs
FP8_MAX = 448.0  # largest value of float8_e4m3fn
MAX_NORM = 1.0


def listed():
    return [
        # one token of a sequence that is being written: latency alone
        dict(name="rotary_one_token", op="rotary", rows=1, heads=28, kv=4, dim=128, sections="16,24,24", cycle=False, pairing="halves",
             inverse=False, dtype="bfloat16", base=1e6, start=30000),
        # a packed microbatch at its full budget; queries and keys lie in the rows of one projection
        dict(name="rotary_microbatch", op="rotary", rows=32768, heads=28, kv=4, dim=128, sections="16,24,24", cycle=False, pairing="halves",
             inverse=False, dtype="bfloat16", base=1e6, start=0),
        # the backward pass of an odd batch in 32 bits, neighbouring elements paired, the axes in turn, part of the head turned
        dict(name="rotary_grad_ragged", op="rotary", rows=4099, heads=5, kv=1, dim=96, sections="11,11,10", cycle=True, pairing="pairs",
             inverse=True, dtype="float32", base=1e4, start=250000),
        # one token, quantised for an 8-bit product: latency alone
        dict(name="rms_one_row", op="rms", rows=1, cols=3584, dtype="bfloat16", residual=True, bits8=True),
        # a layer's norm over a microbatch at its full budget, the residual stream added on the way
        dict(name="rms_microbatch", op="rms", rows=32768, cols=3584, dtype="bfloat16", residual=True, bits8=False),
        # an odd batch of odd width in 32 bits, no residual
        dict(name="rms_grad_ragged", op="rms_grad", rows=4099, cols=1023, dtype="float32", residual=False),
        # the backward pass of a full microbatch
        dict(name="rms_grad_microbatch", op="rms_grad", rows=32768, cols=3584, dtype="bfloat16", residual=True),
        # a block's 16-bit gradients and odd-sized extras, back to back in one buffer
        dict(name="grad_norm_ragged", op="grad_norm", sizes="1605632,1835008,1001,3584,3584,17,524287", dtype="bfloat16", align=1),
        # the embedding table and its norm in 32 bits
        dict(name="grad_norm_table", op="grad_norm", sizes="117440512,3584,3584", dtype="float32", align=128),
        # the next token of a few sequences: the weights are read once, nothing else counts
        dict(name="logprobs_few_rows", op="logprobs", rows=24, hidden=1024, vocab=32768, valid=1.0, top=8),
        # odd sizes everywhere: the tail of a batch against a vocabulary that no tile divides
        dict(name="logprobs_ragged", op="logprobs", rows=1777, hidden=4104, vocab=50021, valid=0.9, top=20),
        # scoring of a microbatch whose image placeholders (a third here) have no token
        dict(name="logprobs_microbatch", op="logprobs", rows=16384, hidden=3584, vocab=32768, valid=0.66, top=8),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _width(rng, low):
    """A width that a 16-byte access divides (8 elements of 16 bits), none of the round ones."""
    c = 8 * _log_int(rng, low, 1024)
    return c + 8 if c % 1024 == 0 else c


def draw(rng):
    op = rng.choice(["rotary", "rms", "rms_grad", "grad_norm", "logprobs", "logprobs"])
    if op == "rotary":
        dim = rng.choice([64, 80, 96, 128, 128, 256])
        heads = rng.choice([1, 5, 8, 12, 28, 32])
        kv = rng.choice([k for k in (1, 2, 4, 8, heads) if heads % k == 0])
        rows = min(_log_int(rng, 1, 65536), 32768 * 32 * 128 // ((heads + kv) * dim))
        pairs = dim // 2 if rng.random() < 0.7 else dim // 4
        t = rng.randint(1, pairs // 2)
        h = (pairs - t) // 2
        return dict(op=op, rows=rows, heads=heads, kv=kv, dim=dim, sections=f"{t},{h},{pairs - t - h}", cycle=rng.random() < 0.5,
                    pairing=rng.choice(["halves", "pairs"]), inverse=rng.random() < 0.5, dtype=rng.choice(["bfloat16", "bfloat16", "float32"]),
                    base=rng.choice([1e4, 5e5, 1e6]), start=rng.choice([0, _log_int(rng, 100, 1000000)]))
    if op in ("rms", "rms_grad"):
        cols = rng.choice([1024, 3584, 4096, 8192, _log_int(rng, 40, 8191) | 1, _width(rng, 8)])
        dtype = rng.choice(["bfloat16", "bfloat16", "float32"])
        rows = min(_log_int(rng, 1, 131072), 32768 * 3584 // cols // (1 if dtype == "bfloat16" else 2))
        case = dict(op=op, rows=rows, cols=cols, dtype=dtype, residual=rng.random() < 0.7)
        return dict(case, bits8=rng.random() < 0.4) if op == "rms" else case
    if op == "logprobs":
        hidden = rng.choice([1024, 3584, 4096, _width(rng, 16)])
        vocab = rng.choice([32768, _log_int(rng, 1000, 131072)])
        rows = min(_log_int(rng, 1, 16384), 16384 * 32768 * 3584 // (vocab * hidden), (1 << 29) // vocab)
        return dict(op=op, rows=rows, hidden=hidden, vocab=vocab, valid=rng.choice([1.0, round(rng.uniform(0.2, 1.0), 3)]),
                    top=rng.choice([0, 1, 5, 8, 20]))
    total, sizes = _log_int(rng, 1000, 100_000_000), []
    for _ in range(rng.randint(1, 40)):
        sizes.append(max(1, int(total * rng.uniform(0.01, 0.3))))
        total -= sizes[-1]
        if total < 1:
            break
    return dict(op="grad_norm", sizes=",".join(map(str, sizes)), dtype=rng.choice(["float32", "bfloat16"]), align=rng.choice([1, 128, 128]))


# ---- inputs -----------------------------------------------------------------------------------------------------

def _sizes(case):
    """(sizes, element offset of each tensor in the flat buffer, buffer length)"""
    sizes = [int(s) for s in case["sizes"].split(",")]
    offs, at = [], 0
    for n in sizes:
        offs.append(at)
        at += -(-n // case["align"]) * case["align"]
    return sizes, offs, at


def _valid_rows(case):
    return max(1, round(case["rows"] * case["valid"]))


def _frequencies(case):
    """(radians per position, axis) of each pair of elements"""
    sections = [int(s) for s in case["sections"].split(",")]
    n = sum(sections)
    freqs = [case["base"] ** (-i / n) for i in range(n)]
    if not case["cycle"]:
        return freqs, [a for a, s in enumerate(sections) for _ in range(s)]
    axes, left = [], list(sections)
    for i in range(n):  # t, h, w, t, h, w, ...; an axis that has had its share is passed over
        a = next((i + j) % 3 for j in range(3) if left[(i + j) % 3])
        left[a] -= 1
        axes.append(a)
    return freqs, axes


def _positions(case, g):
    """[3, rows] of text runs and images (grids of 14 x 14 tokens) in turn, counted on from `start`"""
    rows, image = case["rows"], 14 * 14
    at = torch.arange(rows, device="cuda")
    span = at // image
    picture = (span % 2 == 1)
    begin = case["start"] + (span + 1) // 2 * image + span // 2 * 14
    k = at % image
    zero = torch.zeros_like(k)
    p = torch.stack([begin + torch.where(picture, o, k) for o in (zero, k // 14, k % 14)])
    return p.to(torch.int32)


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    op, s = case["op"], {"case": case}
    if op == "rotary":
        r, d = case["rows"], case["dim"]
        t = getattr(torch, case["dtype"])
        # a row of the projection: queries, keys, values
        s["qkv"] = (normal(r, (case["heads"] + 2 * case["kv"]) * d) * torch.exp(0.5 * normal(r, 1))).to(t)
        s["pos"] = _positions(case, g)
    elif op in ("rms", "rms_grad"):
        r, c, t = case["rows"], case["cols"], getattr(torch, case["dtype"])
        # a residual stream: a few columns far larger than the rest, rows of differing scale
        x = normal(r, c) * torch.exp(0.5 * normal(r, 1)) * torch.where(torch.rand(c, device="cuda", generator=g) < 0.01, 8.0, 1.0)
        s["x"] = x.to(t)
        s["weight"] = 1 + 0.1 * normal(c)
        if op == "rms":
            if case["residual"]:
                s["residual"] = (2 * normal(r, c)).to(t)
        else:
            s["rstd"] = (s["x"].double().square().mean(1) + EPS).rsqrt().float()
            s["dy"] = (1e-2 * normal(r, c)).to(t)
            if case["residual"]:
                s["dsum"] = (1e-2 * normal(r, c)).to(t)
    elif op == "grad_norm":
        n = _sizes(case)[2]
        s["grad"] = (1e-3 * torch.exp(1.5 * normal(n)) * normal(n)).to(getattr(torch, case["dtype"]))
    else:
        r, h, v = case["rows"], case["hidden"], case["vocab"]
        # Both factors lie on a grid on which every sum of their products is exact in 32 bits: equal logits are then equal in any
        # order of the sums, and which alternatives are listed, and in which order, is defined.
        step = 2.0 ** math.ceil(math.log2(6 / math.sqrt(h) / 255))  # five standard deviations within eight bits
        w = (torch.round(normal(v, h) * (1.2 / math.sqrt(h)) / step)).clamp_(-255, 255) * step
        u = torch.rand(r, device="cuda", generator=g)
        tokens = (torch.exp(u * math.log(v)) - 1).long().clamp_(0, v - 1)  # token ids with a Zipf-like head
        # the model is sure of some tokens and has no idea of others
        x = normal(r, h) + torch.rand(r, 1, device="cuda", generator=g) * 10 * w[tokens]
        x = (torch.round(x * 16) / 16).clamp_(-15, 15)
        keep = torch.rand(r, device="cuda", generator=g).argsort() < _valid_rows(case)
        s.update(x=x.to(torch.bfloat16), w=w.to(torch.bfloat16), tokens=torch.where(keep, tokens, IGNORE).to(torch.int32))
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
    op, rows = case["op"], case["rows"] if "rows" in case else 0
    # output buffers, tables, and with the library its handle, workspace and lists: a program keeps them from step to step
    if op == "rotary":
        freqs, axes = _frequencies(case)
        s["freqs"], s["axes"] = torch.tensor(freqs, dtype=torch.float64, device="cuda"), torch.tensor(axes, device="cuda")
        s["q"], s["k"] = (s["qkv"].new_empty(rows, n, case["dim"]) for n in (case["heads"], case["kv"]))
    elif op == "rms":
        if case["residual"]:
            s["sum"] = torch.empty_like(s["x"])
        s["rstd"] = torch.empty(rows, device="cuda")
        if case["bits8"]:
            s["q"] = torch.empty(rows, case["cols"], dtype=torch.float8_e4m3fn, device="cuda")
            s["scale"] = torch.empty(rows, -(-case["cols"] // GROUP), device="cuda")
        else:
            s["y"] = torch.empty_like(s["x"])
    elif op == "rms_grad":
        s["dx"], s["dweight"] = torch.empty_like(s["x"]), torch.empty(case["cols"], device="cuda")
    elif op == "grad_norm":
        s["norm"], s["factor"] = torch.empty(2, 1, device="cuda")
    else:
        s["logprob"], s["entropy"] = torch.empty(2, rows, device="cuda")
        if case["top"]:
            s["top_ids"] = torch.empty(rows, case["top"], dtype=torch.int32, device="cuda")
            s["top_logprobs"] = torch.empty(rows, case["top"], device="cuda")
    if own:
        pool, fp = _pool()
        s["pool"], s["fp"] = pool, fp
        code = fp.FT_F32 if case.get("dtype") == "float32" else fp.FT_BF16
        if op == "rotary":
            s["config"] = fp.rotary_config(freqs, axes, case["dim"], interleaved=case["pairing"] == "pairs", inverse=case["inverse"])
            d, e = case["dim"], s["qkv"].element_size()
            width = s["qkv"].shape[1]
            s["tensors"] = (fp.RotaryTensor * 2)(*[
                fp.RotaryTensor(src=s["qkv"].data_ptr() + at * d * e, dst=s[key].data_ptr(), src_row=width, src_head=d, dst_row=n * d,
                                dst_head=d, heads=n, dtype=code)
                for key, at, n in (("q", 0, case["heads"]), ("k", case["heads"], case["kv"]))])
        elif op == "rms_grad":
            s["ws_bytes"] = pool.rms_norm_grad_workspace(rows, case["cols"])
        elif op == "grad_norm":
            sizes, offs, _ = _sizes(case)
            g = s["grad"]
            s["tensors"] = (fp.GradTensor * len(sizes))(*[fp.GradTensor(grad=g.data_ptr() + o * g.element_size(), n=n, dtype=code)
                                                          for n, o in zip(sizes, offs)])
            s["ws_bytes"] = pool.grad_norm_workspace()
        elif op == "logprobs":
            s["ws_bytes"] = pool.token_logprobs_workspace(rows, case["hidden"], case["vocab"], case["top"])[1]
        if s.get("ws_bytes"):
            s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------

def _plain_rotary(s):
    case = s["case"]
    r, d, h, kv = case["rows"], case["dim"], case["heads"], case["kv"]
    angle = s["pos"].double()[s["axes"]].T * s["freqs"]
    if case["inverse"]:
        angle = -angle
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    n = cos.shape[2]
    out = {}
    for key, at, heads in (("q", 0, h), ("k", h, kv)):
        x = s["qkv"][:, at * d:(at + heads) * d].view(r, heads, d).float()
        a, b = (x[..., :n], x[..., n:2 * n]) if case["pairing"] == "halves" else (x[..., 0:2 * n:2], x[..., 1:2 * n:2])
        a, b = a * cos - b * sin, a * sin + b * cos
        turned = torch.cat([a, b], -1) if case["pairing"] == "halves" else torch.stack([a, b], -1).flatten(-2)
        out[key] = torch.cat([turned, x[..., 2 * n:]], -1).to(s["qkv"].dtype)
    return out


def _plain_rms(s):
    t = s["x"].dtype
    x = s["x"].float()
    out = {}
    if "residual" in s:
        x = x + s["residual"].float()
        out["sum"] = x.to(t)
    rstd = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    out["rstd"] = rstd[:, 0]
    y = x * rstd * s["weight"]
    if not s["case"]["bits8"]:
        out["y"] = y.to(t)
        return out
    rows, cols = y.shape
    groups = torch.nn.functional.pad(y, (0, -cols % GROUP)).view(rows, -1, GROUP)
    scale = groups.abs().amax(2) / FP8_MAX
    q = groups / torch.where(scale > 0, scale, 1.0)[..., None]
    out["q"] = q.clamp(-FP8_MAX, FP8_MAX).reshape(rows, -1)[:, :cols].to(torch.float8_e4m3fn)
    out["scale"] = scale
    return out


def _plain_rms_grad(s):
    rstd, dy = s["rstd"][:, None], s["dy"].float()
    xhat = s["x"].float() * rstd
    a = dy * s["weight"]
    dx = rstd * (a - xhat * (a * xhat).mean(1, keepdim=True))
    if "dsum" in s:
        dx = dx + s["dsum"].float()
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xhat).sum(0)}


def _plain_grad_norm(s):
    sizes, offs, _ = _sizes(s["case"])
    total = sum(s["grad"][o:o + n].double().square().sum() for n, o in zip(sizes, offs))
    norm = total.sqrt()
    factor = torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)
    return {"norm": norm.float()[None], "factor": factor.float()[None]}


def _plain_logprobs(s):
    top, valid = s["case"]["top"], s["tokens"] >= 0
    token = torch.where(valid, s["tokens"], 0).long()[:, None]
    x = torch.where(valid[:, None], s["x"].float(), 0.0)
    z = x @ s["w"].float().T
    out = {}
    if top:
        # ordered by value and, where values are equal, by id: one whole number a logit, its bits in the order of the values above the id's complement
        bits = z.view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = key.mul_(1 << 32).add_((1 << 32) - 1 - torch.arange(z.shape[1], device="cuda"))
        ids = (1 << 32) - 1 - (key.topk(min(top, z.shape[1]), 1).values & ((1 << 32) - 1))
        del key
        picks = z.gather(1, ids)
    most = z.max(1, keepdim=True).values
    picked = z.gather(1, token)
    z = z.sub_(most)
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    entropy = log_total - (e.mul_(z)).sum(1, keepdim=True) / total
    lse = most + log_total
    out["logprob"] = torch.where(valid, (picked - lse)[:, 0], 0.0)
    out["entropy"] = torch.where(valid, entropy[:, 0], 0.0)
    if top:
        out["top_ids"] = torch.where(valid[:, None], ids, -1).to(torch.int32)
        out["top_logprobs"] = torch.where(valid[:, None], picks - lse, 0.0)
    return out


_PLAIN = {"rotary": _plain_rotary, "rms": _plain_rms, "rms_grad": _plain_rms_grad, "grad_norm": _plain_grad_norm, "logprobs": _plain_logprobs}


# ---- the library's calls ----------------------------------------------------------------------------------------

def _own(s):
    case, pool, fp = s["case"], s["pool"], s["fp"]
    op, st = case["op"], torch.cuda.current_stream().cuda_stream
    p = {k: t.data_ptr() for k, t in s.items() if isinstance(t, torch.Tensor)}
    code = fp.FT_F32 if case.get("dtype") == "float32" else fp.FT_BF16
    if op == "rotary":
        rc = pool.rotary(case["rows"], p["pos"], case["rows"], s["config"], s["tensors"], st)
        out = ("q", "k")
    elif op == "rms":
        c, b8 = case["cols"], case["bits8"]
        groups = -(-c // GROUP)
        rc = pool.rms_norm(case["rows"], c, p["x"], c, p.get("residual", 0), c, code, p["weight"], fp.FT_F32, EPS, p.get("sum", 0), c,
                           p.get("y", 0), c, p.get("q", 0), c, p.get("scale", 0), groups, p["rstd"], st)
        out = (("sum",) if case["residual"] else ()) + ("rstd",) + (("q", "scale") if b8 else ("y",))
    elif op == "rms_grad":
        c = case["cols"]
        rc = pool.rms_norm_grad(case["rows"], c, p["dy"], c, p["x"], c, p.get("dsum", 0), c, code, p["weight"], fp.FT_F32, p["rstd"],
                                p["dx"], c, p["dweight"], False, p["ws"], s["ws_bytes"], st)
        out = ("dx", "dweight")
    elif op == "grad_norm":
        rc = pool.grad_norm(s["tensors"], MAX_NORM, 0, 0, p["norm"], p["factor"], p["ws"], s["ws_bytes"], st)
        out = ("norm", "factor")
    else:
        h = case["hidden"]
        rc = pool.token_logprobs(case["rows"], h, case["vocab"], p["x"], h, p["w"], h, p["tokens"], 1.0, p["logprob"], p["entropy"],
                                 case["top"], p.get("top_ids", 0), p.get("top_logprobs", 0), p["ws"], s["ws_bytes"], st)
        out = ("logprob", "entropy") + (("top_ids", "top_logprobs") if case["top"] else ())
    if rc:
        raise fp.FlowpoolError(rc, op)
    return {k: s[k] for k in out}


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state["case"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    e = 4 if case.get("dtype") == "float32" else 2
    if op == "rotary":
        n = case["rows"] * (case["heads"] + case["kv"]) * case["dim"]
        return {"bytes": 2 * n * e + 12 * case["rows"], "flops": 3 * n}
    if op == "rms":
        r, c = case["rows"], case["cols"]
        each = (1 + 2 * case["residual"]) * e + (1 + 4 / GROUP if case["bits8"] else e)
        return {"bytes": r * c * each + 4 * c + 4 * r, "flops": (5 + case["residual"]) * r * c}
    if op == "rms_grad":
        r, c = case["rows"], case["cols"]
        return {"bytes": r * c * e * (4 if case["residual"] else 3) + 8 * c + 4 * r, "flops": (9 + case["residual"]) * r * c}
    if op == "grad_norm":
        n = sum(_sizes(case)[0])
        return {"bytes": e * n + 8, "flops": 2 * n}
    n, r, h, v = _valid_rows(case), case["rows"], case["hidden"], case["vocab"]
    return {"bytes": 2 * n * h + 2 * v * h + 12 * r + 8 * r * case["top"], "flops": 2 * n * h * v}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    d = {k: t.double() for k, t in s.items() if isinstance(t, torch.Tensor) and t.is_floating_point()}
    op = case["op"]
    if op == "rotary":
        freqs, axes = _frequencies(case)
        n, dim, at, out = len(freqs), case["dim"], 0, {}
        # each pair as a complex number, turned by a unit one
        turn = torch.stack([s["pos"][a].double() * f for f, a in zip(freqs, axes)], 1) * (-1 if case["inverse"] else 1)
        turn = torch.polar(torch.ones_like(turn), turn)[:, None]
        first = torch.arange(n, device="cuda") * (1 if case["pairing"] == "halves" else 2)
        second = first + (n if case["pairing"] == "halves" else 1)
        for key, heads in (("q", case["heads"]), ("k", case["kv"])):
            x = d["qkv"][:, at:at + heads * dim].reshape(-1, heads, dim).clone()
            at += heads * dim
            z = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = z.real, z.imag
            out[key] = x
        return out
    if op == "rms":
        x, out = d["x"], {}
        if case["residual"]:
            x = out["sum"] = x + d["residual"]
        out["rstd"] = (torch.einsum("rc,rc->r", x, x) / case["cols"] + EPS) ** -0.5
        y = torch.einsum("rc,r,c->rc", x, out["rstd"], d["weight"])
        if not case["bits8"]:
            return dict(out, y=y)
        group = torch.arange(case["cols"], device="cuda") // GROUP
        top = torch.zeros(case["rows"], int(group[-1]) + 1, dtype=torch.float64, device="cuda")
        top.scatter_reduce_(1, group.expand_as(y), y.abs(), "amax")
        v = y * (FP8_MAX / torch.where(top > 0, top, 1.0))[:, group]
        # the nearest value of the format: 3 bits behind the leading one, multiples of 2^-9 below 2^-6
        unit = 2.0 ** (torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
        return dict(out, q=torch.round(v / unit) * unit, scale=top / FP8_MAX)
    if op == "rms_grad":
        # dx = J^T (w dy), J = rstd (I - xhat xhat^T / c)
        a, r = d["dy"] * d["weight"], d["rstd"][:, None]
        along = torch.einsum("rc,rc->r", a, d["x"])[:, None] * r ** 2 / case["cols"]
        dx = (a - along * d["x"]) * r
        return {"dx": dx + d["dsum"] if case["residual"] else dx, "dweight": torch.einsum("rc,rc,r->c", d["dy"], d["x"], d["rstd"])}
    if op == "grad_norm":
        sizes, offs, _ = _sizes(case)
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(d["grad"][o:o + n]) for n, o in zip(sizes, offs)]))
        return {"norm": norm[None], "factor": torch.clamp(MAX_NORM / norm, max=1.0)[None]}
    r, top = case["rows"], case["top"]
    rows = torch.nonzero(s["tokens"] != IGNORE)[:, 0]
    y = s["tokens"][rows].long()
    z = torch.mm(d["x"][rows], d["w"].T)
    best = z.topk(min(top, case["vocab"]), 1).values if top else None
    picked = z[torch.arange(len(y), device="cuda"), y]
    lse = torch.logsumexp(z, 1)
    z -= lse[:, None]
    entropy = -torch.einsum("rv,rv->r", z.exp(), z)

    def whole(v):
        return torch.zeros(r, *v.shape[1:], dtype=torch.float64, device="cuda").index_copy(0, rows, v)
    out = {"logprob": whole(picked - lse), "entropy": whole(entropy)}
    if top:
        out.update(top_ids=None, top_logprobs=whole(best - lse[:, None]))
    return out
