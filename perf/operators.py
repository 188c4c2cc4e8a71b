"""The operators of a gated recurrent block and of its training step, as they are called, beside their plain forms.

  norm       root-mean-square norm over features that P workers share, with the residual's addition before it; y in the
             tensor's type, or in 8 bits with a scale for each block of 128 features; and its adjoint
  linear8    products of 8-bit operands with a scale for each block of 128 along the sum: the forward pass of a
             partitioned layer, and its whole adjoint from bf16 tensors on (quantisation of dy and x, dx, dW)
  scan       h_t = a_t h_{t-1} + u_t over time that P workers share, its adjoint, and the step of single tokens
  adamw      the update of many arrays at once, states in 32 bits or in 8

8-bit numbers are e4m3 with a power of two (e8m0) for each block: the block's largest magnitude is at most 448 times it.
A case is a flat dict.  listed() names twelve, draw() gives more of the same ranges, exact() computes what run() returns
in 64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 128
EPS = 1e-6


# ---------------------------------------------------------------- cases

def _norm(dtype, rows, n_f, parts, back=False, q8=False, residual=True, **name):
    return dict(kind="norm_bwd" if back else "norm_fwd", dtype=dtype, rows=rows, n_f=n_f, parts=parts, q8=q8,
                residual=residual, **name)


def _linear(dtype, n_b, n_fi, n_fo, p_fo, p_fi, back=False, **name):
    return dict(kind="linear8_bwd" if back else "linear8_fwd", dtype=dtype, n_b=n_b, n_fi=n_fi, n_fo=n_fo, p_fo=p_fo,
                p_fi=p_fi, **name)


def _scan(dtype, n_b, steps, n_c, parts, gate, back=False, ragged=False, **name):
    return dict(kind="scan_bwd" if back else "scan_fwd", dtype=dtype, n_b=n_b, steps=steps, n_c=n_c, parts=parts,
                gate=gate, ragged=ragged, **name)


def listed():
    return [
        # decoding: the norm before a block for four tokens at a time, answered in the 8 bits that the next product reads
        _norm("bf16", 4, 4096, 1, q8=True, name="norm_token"),
        # the same before a block in training, a batch of 8192 tokens, features on two workers
        _norm("bf16", 8192, 4096, 2, q8=True, name="norm_q8"),
        # the norm's adjoint with a width and a batch that nothing divides, over three workers
        _norm("f32", 5003, 2000, 3, back=True, name="norm_bwd_odd"),
        # decoding: the wide dense layer of the configurations for eight tokens, all of it reading weights
        _linear("bf16", 8, 4096, 4096, 1, 1, name="linear8_token"),
        # that layer at its batch, on its 2 x 2 workers
        _linear("bf16", 256, 4096, 4096, 2, 2, name="linear8_4096"),
        # a classifier's last layer with an odd batch and an odd number of classes: rows of 666 and 667 bytes
        _linear("f32", 37, 2000, 1001, 2, 3, name="linear8_head"),
        # a training step's adjoint for 8192 tokens, from bf16 gradients and activations on; the largest case
        _linear("bf16", 8192, 4096, 4096, 1, 1, back=True, name="linear8_bwd"),
        # one long sequence on four workers, few channels: time has to be split to fill the card
        _scan("bf16", 1, 65536, 1024, 4, "sigmoid", name="scan_long"),
        # the adjoint for a ragged batch (one sequence is empty), odd sizes
        _scan("f32", 7, 2049, 1001, 3, "sigmoid", back=True, ragged=True, name="scan_bwd_ragged"),
        # decoding: one step of 64 sequences whose states lie in a pool of slots
        dict(kind="scan_step", dtype="bf16", rows=64, n_c=4096, slots=96, gate="sigmoid", name="scan_step"),
        # the weights of the small convolutional network: ten arrays, 60 to 24000 numbers, latency only
        dict(kind="adamw", shapes="6x25,6,16x150,16,120x400,120,84x120,84,10x84,10", g="f32", states="f32", copy=False,
             name="adamw_cnn"),
        # recurrent blocks with states in 8 bits: products of 2048 features and gains, 170 million weights
        dict(kind="adamw", shapes=",".join(["2048x2048,2048x2048,8192x2048,2048x8192,2048"] * 4), g="bf16", states="8bit",
             copy=True, name="adamw_8bit"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm_fwd", "norm_bwd", "linear8_fwd", "linear8_bwd", "scan_fwd", "scan_bwd", "scan_step", "adamw"])
    dtype = rng.choice(["f32", "bf16"])
    even = lambda n: n if rng.random() < 0.5 else max(128, n // 128 * 128)  # noqa: E731
    gate = rng.choice(["given", "sigmoid"])
    while True:
        if kind.startswith("norm"):
            rows, n_f = _log(rng, 1, 20000), even(_log(rng, 64, 8192))
            if rows * n_f <= 1 << 26:
                return _norm(dtype, rows, n_f, rng.choice([1, 1, 2, 3, 4]), kind == "norm_bwd", rng.random() < 0.5, rng.random() < 0.7)
        elif kind.startswith("linear8"):
            n_b, n_fi, n_fo = _log(rng, 1, 8192), even(_log(rng, 64, 8192)), even(_log(rng, 64, 8192))
            if n_b * n_fi * n_fo <= 1 << 36:
                return _linear(dtype, n_b, n_fi, n_fo, rng.choice([1, 1, 2, 3]), rng.choice([1, 1, 2, 3]), kind == "linear8_bwd")
        elif kind == "scan_step":
            rows = _log(rng, 1, 512)
            return dict(kind=kind, dtype=dtype, rows=rows, n_c=even(_log(rng, 64, 8192)), slots=rows + rng.randrange(64), gate=gate)
        elif kind.startswith("scan"):
            n_b, steps, n_c = _log(rng, 1, 64), _log(rng, 4, 65536), even(_log(rng, 64, 8192))
            if n_b * steps * n_c <= 1 << 26:
                return _scan(dtype, n_b, steps, n_c, rng.choice([1, 1, 2, 3, 4]), gate, kind == "scan_bwd", rng.random() < 0.5)
        else:
            n, most = rng.randrange(1, 40), _log(rng, 64, 1 << 21)
            shapes = ["%d" % max(1, int(most * rng.random() ** 3)) for _ in range(n)]
            return dict(kind="adamw", shapes=",".join(shapes), g=dtype, states=rng.choice(["f32", "8bit"]), copy=rng.random() < 0.5)


# ---------------------------------------------------------------- pieces of the plain forms

def _parts(n, parts):
    return [n // parts + (r < n % parts) for r in range(parts)]


def _cut(x, parts, dim):
    return [t.contiguous() for t in x.split(_parts(x.shape[dim], parts), dim)]


def _rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _byte(amax):
    """The biased exponent of the smallest power of two that 448 times of is at least amax; never a subnormal one."""
    bits = amax.view(torch.int32)
    byte = (((bits + 0x1FFFFF) >> 23) - 8).clamp(min=1)
    return torch.where(bits >= 0x7F800000, torch.full_like(byte, 255), byte)


def _power(byte):
    return (byte << 23).view(torch.float32)


def _as_scale(byte):
    return byte.to(torch.uint8).view(torch.float8_e8m0fnu)


def _blocks(x):
    """[rows, columns] as [rows, blocks, 128], zeros behind the end."""
    return torch.nn.functional.pad(x, (0, -x.shape[1] % BLOCK)).view(x.shape[0], -1, BLOCK)


def _quant_rows(x):
    """e4m3 numbers of fp32 [rows, columns] and the scales [blocks, rows]."""
    b = _blocks(x)
    byte = _byte(b.abs().amax(2))
    q = (b * _power(254 - byte)[:, :, None]).view(x.shape[0], -1)[:, :x.shape[1]]
    return q.to(torch.float8_e4m3fn).contiguous(), _as_scale(byte.t().contiguous())


def _quant_tiles(x):
    """e4m3 numbers of fp32 [rows, columns] and one scale for each tile of 128 x 128."""
    r, c = x.shape
    t = torch.nn.functional.pad(x, (0, -c % BLOCK, 0, -r % BLOCK)).view(-(-r // BLOCK), BLOCK, -1, BLOCK)
    byte = _byte(t.abs().amax(3).amax(1))
    q = (t * _power(254 - byte)[:, None, :, None]).view(-(-r // BLOCK) * BLOCK, -1)[:r, :c]
    return q.to(torch.float8_e4m3fn).contiguous(), _as_scale(byte)


def _value(s):
    return _power(s.view(torch.uint8).to(torch.int32))


def _of_rows(q, s):
    return q.float() * _value(s).t().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _of_tiles(q, s):
    return q.float() * _value(s).repeat_interleave(BLOCK, 0)[:q.shape[0]].repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _running(a, b):
    """All h_t = a_t h_{t-1} + b_t of [n, steps, channels] in log2(steps) rounds, each of which doubles the reach."""
    reach = 1
    while reach < a.shape[1]:
        b = torch.cat([b[:, :reach], b[:, reach:] + a[:, reach:] * b[:, :-reach]], 1)
        a = torch.cat([a[:, :reach], a[:, reach:] * a[:, :-reach]], 1)
        reach *= 2
    return b


def _inside(s, steps):
    """[n, steps, 1]: whether a step lies inside its sequence."""
    return (torch.arange(steps, device="cuda")[None] < s["lengths"][:, None])[:, :, None]


# ---------------------------------------------------------------- norm

def _prepare_norm(c, gen, s):
    t, P = TYPES[c["dtype"]], c["parts"]
    rows, n_f = c["rows"], c["n_f"]
    loud = torch.where(torch.rand(n_f, generator=gen, device="cuda") < 0.01, 20.0, 1.0)  # a residual stream has loud features
    s["gain"] = _cut(1 + 0.1 * _rand(gen, n_f), P, 0)
    new = lambda like, kind: [torch.empty(v.shape, dtype=kind, device="cuda") for v in like]  # noqa: E731
    if c["kind"] == "norm_fwd":
        s["x"] = _cut(_rand(gen, rows, n_f).to(t), P, 1)
        s["res"] = _cut((3 * loud * _rand(gen, rows, n_f)).to(t), P, 1) if c["residual"] else None
        s["sum"] = new(s["x"], t) if c["residual"] else None
        s["rstd"] = torch.empty(rows, device="cuda")
        s["y"] = None if c["q8"] else new(s["x"], t)
        s["q"] = new(s["x"], torch.float8_e4m3fn) if c["q8"] else None
        s["qs"] = [torch.empty(-(-v.shape[1] // BLOCK), rows, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
                   for v in s["x"]] if c["q8"] else None
    else:
        x = (3 * loud * _rand(gen, rows, n_f)).to(t)
        s["rstd"] = torch.rsqrt(x.float().square().mean(1) + EPS)
        s["x"] = _cut(x, P, 1)
        s["dy"] = _cut((1e-3 * _rand(gen, rows, n_f)).to(t), P, 1)
        s["dsum"] = _cut((1e-3 * _rand(gen, rows, n_f)).to(t), P, 1) if c["residual"] else None
        s["dx"] = new(s["x"], t)
        s["dgain"] = new(s["gain"], torch.float32)
    if own:
        import paper_2006_03108_amd as dd
        s["plan"] = dd.distdl_rmsnorm_plan_create(rows, n_f, P, EPS, t)


def _own_norm(c, s):
    import paper_2006_03108_amd as dd
    if c["kind"] == "norm_fwd":
        dd.distdl_rmsnorm_fwd(s["plan"], s["x"], s["res"], s["gain"], s["sum"], s["y"], s["q"], s["qs"], s["rstd"])
        return {k: s[k] for k in ("sum", "y", "q", "qs", "rstd")}
    dd.distdl_rmsnorm_bwd(s["plan"], s["x"], s["gain"], s["rstd"], s["dy"], s["dsum"], s["dx"], s["dgain"])
    return {"dx": s["dx"], "dgain": s["dgain"]}


def _plain_norm(c, s):
    t, P = TYPES[c["dtype"]], c["parts"]
    x, gain = torch.cat(s["x"], 1).float(), torch.cat(s["gain"])
    if c["kind"] == "norm_fwd":
        if c["residual"]:
            x = x + torch.cat(s["res"], 1).float()
        rstd = torch.rsqrt(x.square().mean(1) + EPS)
        y = _cut(x * rstd[:, None] * gain, P, 1)
        q = [_quant_rows(v) for v in y] if c["q8"] else None
        return {"sum": _cut(x.to(t), P, 1) if c["residual"] else None, "y": None if c["q8"] else [v.to(t) for v in y],
                "q": q and [v[0] for v in q], "qs": q and [v[1] for v in q], "rstd": rstd}
    n = x * s["rstd"][:, None]
    dy = torch.cat(s["dy"], 1).float()
    dn = dy * gain
    dx = (dn - n * (dn * n).mean(1, keepdim=True)) * s["rstd"][:, None]
    if c["residual"]:
        dx = dx + torch.cat(s["dsum"], 1).float()
    return {"dx": _cut(dx.to(t), P, 1), "dgain": _cut((dy * n).sum(0), P, 0)}


def _exact_norm(c, s):
    P = c["parts"]
    x, gain = torch.cat(s["x"], 1).double(), torch.cat(s["gain"]).double()
    if c["kind"] == "norm_fwd":
        if c["residual"]:
            x += torch.cat(s["res"], 1).double()
        rstd = 1 / ((x * x).sum(1) / c["n_f"] + EPS).sqrt()
        y = _cut(torch.einsum("rf,r,f->rf", x, rstd, gain), P, 1)
        q = []
        for v in y if c["q8"] else []:  # the values before they are rounded to 8 bits, in units of their scale
            scale = torch.stack([torch.exp2(torch.ceil(torch.log2(b.abs().amax(1) / 448))) for b in v.split(BLOCK, 1)])
            q.append((torch.cat([b / scale[k][:, None] for k, b in enumerate(v.split(BLOCK, 1))], 1), scale))
        return {"sum": _cut(x, P, 1) if c["residual"] else None, "y": None if c["q8"] else y,
                "q": [v[0] for v in q] if c["q8"] else None, "qs": [v[1] for v in q] if c["q8"] else None, "rstd": rstd}
    dy, r = torch.cat(s["dy"], 1).double(), s["rstd"].double()
    dot = torch.einsum("rf,rf,f->r", dy, x, gain) / c["n_f"]
    dx = r[:, None] * dy * gain - (r ** 3 * dot)[:, None] * x
    if c["residual"]:
        dx += torch.cat(s["dsum"], 1).double()
    return {"dx": _cut(dx, P, 1), "dgain": _cut(torch.einsum("rf,rf,r->f", dy, x, r), P, 0)}


def _work_norm(c):
    n, size = c["rows"] * c["n_f"], 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "norm_fwd":
        return {"bytes": n * ((3 if c["residual"] else 1) * size + (1 + 1 / BLOCK if c["q8"] else size)) + 4 * c["n_f"] + 4 * c["rows"], "flops": 6 * n}
    return {"bytes": n * (4 if c["residual"] else 3) * size + 8 * c["n_f"] + 4 * c["rows"], "flops": 10 * n}


# ---------------------------------------------------------------- linear8

def _prepare_linear(c, gen, s):
    t, n_b, n_fi, n_fo = TYPES[c["dtype"]], c["n_b"], c["n_fi"], c["n_fo"]
    w = [_cut(rows, c["p_fi"], 1) for rows in _cut(_rand(gen, n_fo, n_fi) / math.sqrt(n_fi), c["p_fo"], 0)]
    w = [v for row in w for v in row]  # worker (i, j) at i * p_fi + j
    new = lambda shape, kind: torch.empty(shape, dtype=kind, device="cuda")  # noqa: E731
    fo, fi = _parts(n_fo, c["p_fo"]), _parts(n_fi, c["p_fi"])
    if c["kind"] == "linear8_fwd":
        x = [_quant_rows(v) for v in _cut(_rand(gen, n_b, n_fi), c["p_fi"], 1)]
        s["xq"], s["xs"] = [v[0] for v in x], [v[1] for v in x]
        w = [_quant_tiles(v) for v in w]
        s["wq"], s["ws"] = [v[0] for v in w], [v[1] for v in w]
        s["y"] = [new((n_b, n), t) for n in fo]
    else:
        s["dy"] = _cut((1e-3 * _rand(gen, n_b, n_fo)).to(torch.bfloat16), c["p_fo"], 1)
        s["x"] = _cut(_rand(gen, n_b, n_fi).to(torch.bfloat16), c["p_fi"], 1)
        w = [_quant_tiles(v.t().contiguous()) for v in w]  # the transposed weights of a data gradient
        s["wtq"], s["wts"] = [v[0] for v in w], [v[1] for v in w]
        s["dx"] = [new((n_b, n), t) for n in fi]
        s["dw"] = [new((m, n), torch.float32) for m in fo for n in fi]
        e4, e8, blocks = torch.float8_e4m3fn, torch.float8_e8m0fnu, lambda n: -(-n // BLOCK)  # noqa: E731
        s["dyq"], s["dys"] = [new((n_b, n), e4) for n in fo], [new((blocks(n), n_b), torch.uint8).view(e8) for n in fo]
        s["dytq"], s["dyts"] = [new((n, n_b), e4) for n in fo], [new((blocks(n_b), n), torch.uint8).view(e8) for n in fo]
        s["xtq"], s["xts"] = [new((n, n_b), e4) for n in fi], [new((blocks(n_b), n), torch.uint8).view(e8) for n in fi]
    if own:
        import paper_2006_03108_amd as dd
        s["plan"] = dd.distdl_linear8_plan_create(n_b, n_fi, n_fo, c["p_fo"], c["p_fi"], t)


def _own_linear(c, s):
    import paper_2006_03108_amd as dd
    if c["kind"] == "linear8_fwd":
        dd.distdl_linear8_fwd(s["plan"], s["xq"], s["xs"], s["wq"], s["ws"], s["y"])
        return {"y": s["y"]}
    dd.distdl_quant8(s["dy"], s["dyq"], s["dys"], s["dytq"], s["dyts"])
    dd.distdl_quant8(s["x"], None, None, s["xtq"], s["xts"])
    dd.distdl_linear8_bwd_x(s["plan"], s["dyq"], s["dys"], s["wtq"], s["wts"], s["dx"])
    dd.distdl_linear8_bwd_w(s["plan"], s["dytq"], s["dyts"], s["xtq"], s["xts"], s["dw"])
    return {"dx": s["dx"], "dw": s["dw"]}


def _plain_linear(c, s):
    t, p_fo, p_fi = TYPES[c["dtype"]], c["p_fo"], c["p_fi"]
    if c["kind"] == "linear8_fwd":
        x = torch.cat([_of_rows(q, v) for q, v in zip(s["xq"], s["xs"])], 1)
        w = [_of_tiles(q, v) for q, v in zip(s["wq"], s["ws"])]
        return {"y": [(x @ torch.cat(w[i * p_fi:(i + 1) * p_fi], 1).t()).to(t) for i in range(p_fo)]}
    dyq = torch.cat([_of_rows(*_quant_rows(v.float())) for v in s["dy"]], 1)
    dytq = [_of_rows(*_quant_rows(v.float().t().contiguous())) for v in s["dy"]]
    xtq = [_of_rows(*_quant_rows(v.float().t().contiguous())) for v in s["x"]]
    wt = [_of_tiles(q, v) for q, v in zip(s["wtq"], s["wts"])]
    return {"dx": [(dyq @ torch.cat(wt[j::p_fi], 1).t()).to(t) for j in range(p_fi)],
            "dw": [dy @ x.t() for dy in dytq for x in xtq]}


def _exact_rounded(v):
    """Rows of 64-bit numbers rounded to e4m3 in blocks of 128."""
    out = torch.empty_like(v)
    for k in range(0, v.shape[1], BLOCK):
        b = v[:, k:k + BLOCK]
        scale = torch.exp2(torch.ceil(torch.log2(b.abs().amax(1, keepdim=True).clamp(min=2.0 ** -110) / 448)))
        step = torch.exp2(torch.floor(torch.log2((b / scale).abs().clamp(min=2.0 ** -6))) - 3)
        out[:, k:k + BLOCK] = torch.round(b / scale / step) * step * scale
    return out


def _exact_linear(c, s):
    p_fo, p_fi = c["p_fo"], c["p_fi"]

    def spread(s8, shape, rows, columns):  # the scales at each number, by its indexes
        r, k = torch.arange(shape[0], device="cuda") // rows, torch.arange(shape[1], device="cuda") // columns
        v = torch.exp2(s8.view(torch.uint8).double() - 127)
        return (v if rows > 1 else v.t())[r[:, None], k[None]]

    if c["kind"] == "linear8_fwd":
        x = [q.double() * spread(v, q.shape, 1, BLOCK) for q, v in zip(s["xq"], s["xs"])]
        w = [q.double() * spread(v, q.shape, BLOCK, BLOCK) for q, v in zip(s["wq"], s["ws"])]
        return {"y": [sum(x[j] @ w[i * p_fi + j].t().contiguous() for j in range(p_fi)) for i in range(p_fo)]}
    dy, x = [v.double() for v in s["dy"]], [v.double() for v in s["x"]]
    wt = [q.double() * spread(v, q.shape, BLOCK, BLOCK) for q, v in zip(s["wtq"], s["wts"])]
    dyq = [_exact_rounded(v) for v in dy]
    dyt, xt = [_exact_rounded(v.t().contiguous()) for v in dy], [_exact_rounded(v.t().contiguous()) for v in x]
    return {"dx": [sum(dyq[i] @ wt[i * p_fi + j].t().contiguous() for i in range(p_fo)) for j in range(p_fi)],
            "dw": [a @ b.t().contiguous() for a in dyt for b in xt]}


def _work_linear(c):
    m, k, n, size = c["n_b"], c["n_fi"], c["n_fo"], 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "linear8_fwd":
        return {"bytes": (m * k + n * k) + m * -(-k // BLOCK) + m * n * size, "flops": 2 * m * n * k}
    return {"bytes": 2 * m * n + 2 * m * k + n * k + m * k * size + 4 * n * k, "flops": 4 * m * n * k}


# ---------------------------------------------------------------- scan

def _gates(c, gen, *shape):
    """Gates that remember for tens to hundreds of steps: logits, or values below one."""
    g = 2.5 + 1.5 * _rand(gen, *shape)
    return (g if c["gate"] == "sigmoid" else torch.sigmoid(g)).to(TYPES[c["dtype"]])


def _terms(c, a, x):
    """a_t and u_t in fp32 from what is given."""
    a, x = a.float(), x.float()
    if c["gate"] == "given":
        return a, x
    a = torch.sigmoid(a)
    return a, (1 - a) * x


def _states(c, s):
    """All states in fp32, those behind a sequence's end its last one."""
    a, u = _terms(c, torch.cat(s["a"], 1), torch.cat(s["x"], 1))
    if s["lengths"] is not None:
        inside = _inside(s, c["steps"])
        a, u = torch.where(inside, a, 1.0), torch.where(inside, u, 0.0)
    u[:, 0] += a[:, 0] * s["h0"]
    return _running(a, u)


def _prepare_scan(c, gen, s):
    t, P, n_c = TYPES[c["dtype"]], c.get("parts", 1), c["n_c"]
    if c["kind"] == "scan_step":
        n = c["rows"]
        s["a"], s["x"], s["state"] = _gates(c, gen, n, n_c), _rand(gen, n, n_c).to(t), 0.3 * _rand(gen, c["slots"], n_c)
        slots = torch.randperm(c["slots"], generator=gen, device="cuda")[:n]
        s["slots"] = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.1, -1, slots).to(torch.int32)  # some are idle
        s["h"] = torch.empty_like(s["x"])
        return
    n_b, T = c["n_b"], c["steps"]
    s["a"], s["x"] = _cut(_gates(c, gen, n_b, T, n_c), P, 1), _cut(_rand(gen, n_b, T, n_c).to(t), P, 1)
    s["h0"] = 0.3 * _rand(gen, n_b, n_c)
    s["lengths"] = None
    if c["ragged"]:
        s["lengths"] = torch.randint(0, T + 1, (n_b,), generator=gen, device="cuda", dtype=torch.int32)
        s["lengths"][0], s["lengths"][-1] = T, 0 if n_b > 1 else T
    new = lambda: [torch.empty_like(v) for v in s["x"]]  # noqa: E731
    if c["kind"] == "scan_fwd":
        s["h"], s["hT"] = new(), torch.empty(n_b, n_c, device="cuda")
    else:
        h = _states(c, s)
        if s["lengths"] is not None:
            h = torch.where(_inside(s, T), h, 0.0)
        s["h"] = _cut(h.to(t), P, 1)
        s["dh"], s["dhT"] = _cut(_rand(gen, n_b, T, n_c).to(t), P, 1), _rand(gen, n_b, n_c)
        s["da"], s["dx"], s["dh0"] = new(), new(), torch.empty(n_b, n_c, device="cuda")
    if own:
        import paper_2006_03108_amd as dd
        s["plan"] = dd.distdl_scan_plan_create(n_b, T, n_c, P, c["gate"], t)


def _own_scan(c, s):
    import paper_2006_03108_amd as dd
    if c["kind"] == "scan_step":
        dd.distdl_scan_step(s["a"], s["x"], s["state"], s["slots"], s["h"], c["gate"])
        return {"h": s["h"], "state": s["state"]}
    if c["kind"] == "scan_fwd":
        dd.distdl_scan_fwd(s["plan"], s["a"], s["x"], s["h0"], s["lengths"], s["h"], s["hT"])
        return {"h": s["h"], "hT": s["hT"]}
    dd.distdl_scan_bwd(s["plan"], s["a"], s["x"], s["h"], s["h0"], s["lengths"], s["dh"], s["dhT"], s["da"], s["dx"], s["dh0"])
    return {"da": s["da"], "dx": s["dx"], "dh0": s["dh0"]}


def _plain_scan(c, s):
    t, P = TYPES[c["dtype"]], c.get("parts", 1)
    if c["kind"] == "scan_step":
        a, u = _terms(c, s["a"], s["x"])
        at, live = s["slots"].long().clamp(min=0), (s["slots"] >= 0)[:, None]
        old = s["state"][at]
        h = a * old + u
        s["state"].index_add_(0, at, torch.where(live, h - old, 0.0))
        return {"h": torch.where(live, h, 0.0).to(t), "state": s["state"]}
    T = c["steps"]
    if c["kind"] == "scan_fwd":
        h = _states(c, s)
        hT = h[:, -1].clone()
        if s["lengths"] is not None:
            h = torch.where(_inside(s, T), h, 0.0)
        return {"h": _cut(h.to(t), P, 1), "hT": hT}
    x = torch.cat(s["x"], 1)
    a, _ = _terms(c, torch.cat(s["a"], 1), x)
    x, h, d = x.float(), torch.cat(s["h"], 1).float(), torch.cat(s["dh"], 1).float()
    before = torch.cat([s["h0"][:, None], h[:, :-1]], 1)
    inside = None if s["lengths"] is None else _inside(s, T)
    live = a if inside is None else torch.where(inside, a, 1.0)
    d = d if inside is None else torch.where(inside, d, 0.0)
    d[:, -1] += s["dhT"]
    later = torch.cat([live[:, 1:], torch.ones_like(live[:, :1])], 1)  # the factor between a state and the next one's gradient
    d = _running(later.flip(1), d.flip(1)).flip(1)
    dh0 = live[:, 0] * d[:, 0]
    if inside is not None:
        d = torch.where(inside, d, 0.0)
    da, dx = (d * before, d) if c["gate"] == "given" else (d * (before - x) * a * (1 - a), d * (1 - a))
    return {"da": _cut(da.to(t), P, 1), "dx": _cut(dx.to(t), P, 1), "dh0": dh0}


def _exact_scan(c, s):
    P = c.get("parts", 1)
    gated = c["gate"] == "sigmoid"
    if c["kind"] == "scan_step":
        a, x, state, h = s["a"].double(), s["x"].double(), s["state"].double(), torch.zeros_like(s["x"], dtype=torch.float64)
        a = 1 / (1 + torch.exp(-a)) if gated else a
        for row, slot in enumerate(s["slots"].tolist()):
            if slot >= 0:
                h[row] = a[row] * state[slot] + ((1 - a[row]) * x[row] if gated else x[row])
                state[slot] = h[row]
        return {"h": h, "state": state}
    n_b, T, n_c = c["n_b"], c["steps"], c["n_c"]
    a, x = torch.cat(s["a"], 1).double(), torch.cat(s["x"], 1).double()
    a = 1 / (1 + torch.exp(-a)) if gated else a
    ends = torch.full((n_b,), T, device="cuda") if s["lengths"] is None else s["lengths"]
    state, zero = s["h0"].double(), torch.zeros(n_b, n_c, dtype=torch.float64, device="cuda")
    if c["kind"] == "scan_fwd":
        h = torch.empty_like(x)
        for t in range(T):
            now = (ends > t)[:, None]
            state = torch.where(now, a[:, t] * state + ((1 - a[:, t]) * x[:, t] if gated else x[:, t]), state)
            h[:, t] = torch.where(now, state, zero)
        return {"h": _cut(h, P, 1), "hT": state}
    h, dh = torch.cat(s["h"], 1).double(), torch.cat(s["dh"], 1).double()
    da, dx, back = torch.empty_like(x), torch.empty_like(x), s["dhT"].double()
    for t in range(T - 1, -1, -1):
        now = (ends > t)[:, None]
        d = back + dh[:, t]
        before = h[:, t - 1] if t else state
        slope = (before - x[:, t]) * a[:, t] * (1 - a[:, t]) if gated else before
        da[:, t], dx[:, t] = torch.where(now, d * slope, zero), torch.where(now, d * (1 - a[:, t]) if gated else d, zero)
        back = torch.where(now, d * a[:, t], back)
    return {"da": _cut(da, P, 1), "dx": _cut(dx, P, 1), "dh0": back}


def _work_scan(c):
    size = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "scan_step":
        n = c["rows"] * c["n_c"]
        return {"bytes": n * (3 * size + 8), "flops": 5 * n}
    n, ends = c["n_b"] * c["steps"] * c["n_c"], c["n_b"] * c["n_c"]
    share = 0.5 if c["ragged"] else 1.0  # steps behind a sequence's end need not be read, but are written; half of them in the mean
    if c["kind"] == "scan_fwd":
        return {"bytes": n * size * (2 * share + 1) + 8 * ends, "flops": 5 * n}
    return {"bytes": n * size * ((4 if c["gate"] == "sigmoid" else 3) * share + 2) + 12 * ends, "flops": 9 * n}


# ---------------------------------------------------------------- adamw

HYPER = dict(lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, step=100, seed=1234)


def _counts(c):
    return [math.prod(int(v) for v in t.split("x")) for t in c["shapes"].split(",")]


def _prepare_adamw(c, gen, s):
    counts = _counts(c)
    starts, at = [], 0
    for n in counts:  # arrays of one allocation, each at a multiple of 128
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    inside = torch.zeros(at, device="cuda")
    for k, n in zip(starts, counts):
        inside[k:k + n] = 1
    loud = torch.exp(_rand(gen, at // BLOCK)).repeat_interleave(BLOCK)  # rows of a gradient differ in size
    s["p"] = 0.02 * _rand(gen, at) * inside
    s["g"] = (1e-3 * loud * _rand(gen, at) * inside).to(TYPES[c["g"]])
    m, v = 3e-4 * loud * _rand(gen, at) * inside, (1e-3 * loud * (0.1 + torch.rand(at, generator=gen, device="cuda"))).square() * inside
    s["p16"] = torch.zeros(at, dtype=torch.bfloat16, device="cuda") if c["copy"] else None
    s["gscale"] = torch.full((1,), 0.8, device="cuda")  # what clipping by the whole gradient's norm left on the device
    s["ms"] = s["vs"] = None
    if c["states"] == "8bit":
        (m, s["ms"]), (v, s["vs"]) = (tuple(t.view(-1) for t in _quant_rows(t.view(1, -1))) for t in (m, v.sqrt()))
    s["m"], s["v"] = m, v
    cut = lambda t, unit: None if t is None else [t[k // unit:k // unit + -(-n // unit)] for k, n in zip(starts, counts)]  # noqa: E731
    s["arrays"] = {k: cut(s[k], BLOCK if k in ("ms", "vs") else 1) for k in ("p", "g", "m", "v", "ms", "vs", "p16")}
    if own:
        import paper_2006_03108_amd as dd
        s["plan"] = dd.distdl_adamw_plan_create(counts, TYPES[c["g"]], c["states"] == "8bit")


def _own_adamw(c, s):
    import paper_2006_03108_amd as dd
    dd.distdl_adamw_step(s["plan"], **s["arrays"], **HYPER, gscale=s["gscale"])
    return {k: s[k] for k in ("p", "m", "v", "ms", "vs", "p16")}


def _noise(n):
    """16 random bits for the first and 16 for the second moment of each of n numbers, from the seed, the step and the place."""
    mask = 0xFFFFFFFF
    key = (HYPER["seed"] * 0x6A09E667 + HYPER["step"] * 0xBB67AE85) & mask
    x = (torch.arange(n, device="cuda") * 0x9E3779B1 + key) & mask
    x = ((x ^ (x >> 15)) * 0x6A09E667) & mask
    x = ((x ^ (x >> 13)) * 0xBB67AE85) & mask
    x = x ^ (x >> 16)
    return (x >> 16).to(torch.int32), (x & 0xFFFF).to(torch.int32)


def _quant_noisy(x, noise, least):
    """e4m3 numbers of x, rounded up or down at random, so that their mean is x; least: what is not zero stays so."""
    b = x.view(-1, BLOCK)
    byte = _byte(b.abs().amax(1))
    y = (b * _power(254 - byte)[:, None]).view(-1)
    size = y.abs()
    small = size < 2.0 ** -6  # (e4m3's subnormal numbers are as far apart as those from 2^-6 on)
    size = torch.where(small, size + 2.0 ** -6, size)
    size = ((size.view(torch.int32) + (noise << 4)) & ~0xFFFFF).view(torch.float32)
    size = torch.where(small, size - 2.0 ** -6, size)
    if least:
        size = torch.where(y > 0, size.clamp(min=2.0 ** -9), size)
    return torch.copysign(size, y).to(torch.float8_e4m3fn), _as_scale(byte)


def _plain_adamw(c, s):
    h, eight = HYPER, c["states"] == "8bit"
    g = s["g"].float() * s["gscale"]
    m, v = s["m"], s["v"]
    if eight:
        m = m.float() * _value(s["ms"]).repeat_interleave(BLOCK)
        v = (v.float() * _value(s["vs"]).repeat_interleave(BLOCK)).square()
    m = m * h["beta1"] + g * (1 - h["beta1"])
    v = v * h["beta2"] + g * g * (1 - h["beta2"])
    root = v.sqrt()
    rate, grow = h["lr"] / (1 - h["beta1"] ** h["step"]), 1 / math.sqrt(1 - h["beta2"] ** h["step"])
    s["p"].copy_(s["p"] * (1 - h["lr"] * h["weight_decay"]) - m / (root * grow + h["eps"]) * rate)
    if eight:
        first, second = _noise(m.numel())
        (m, ms), (v, vs) = _quant_noisy(m, first, False), _quant_noisy(root, second, True)
        s["ms"].copy_(ms)
        s["vs"].copy_(vs)
    s["m"].copy_(m)
    s["v"].copy_(v)
    if c["copy"]:
        s["p16"].copy_(s["p"])
    return {k: s[k] for k in ("p", "m", "v", "ms", "vs", "p16")}


def _exact_adamw(c, s):
    h, eight = HYPER, c["states"] == "8bit"
    out = {k: [] for k in ("p", "m", "v", "ms", "vs")}
    for k in range(0, s["p"].numel(), 1 << 24):  # (a part at a time: 64-bit numbers of the whole are large)
        part = slice(k, k + (1 << 24))
        p, g, m, v = (s[n][part].double() for n in ("p", "g", "m", "v"))
        g *= float(s["gscale"])
        if eight:
            of = slice(k // BLOCK, (k + (1 << 24)) // BLOCK)
            by = lambda t: torch.exp2(t[of].view(torch.uint8).double() - 127)[:, None]  # noqa: E731
            m, v = (m.view(-1, BLOCK) * by(s["ms"])).view(-1), ((v.view(-1, BLOCK) * by(s["vs"])) ** 2).view(-1)
        m = h["beta1"] * m + (1 - h["beta1"]) * g
        v = h["beta2"] * v + (1 - h["beta2"]) * g ** 2
        hat, root = m / (1 - h["beta1"] ** h["step"]), (v / (1 - h["beta2"] ** h["step"])) ** 0.5
        out["p"].append(p - h["lr"] * (hat / (root + h["eps"]) + h["weight_decay"] * p))
        for name, t in (("m", m), ("v", v ** 0.5)) if eight else ():  # in units of the scale, before they are rounded
            t = t.view(-1, BLOCK)
            scale = torch.exp2(torch.ceil(torch.log2(t.abs().amax(1).clamp(min=2.0 ** -110) / 448)).clamp(min=-126))
            out[name].append((t / scale[:, None]).view(-1))
            out[name + "s"].append(scale)
        if not eight:
            out["m"].append(m)
            out["v"].append(v)
    out = {k: torch.cat(v) if v else None for k, v in out.items()}
    return {**out, "p16": out["p"] if c["copy"] else None}


def _work_adamw(c):
    n = sum(_counts(c))
    return {"bytes": n * (8 + (4 if c["g"] == "f32" else 2) + (16 if c["states"] == "f32" else 4 + 4 / BLOCK) + (2 if c["copy"] else 0)), "flops": 16 * n}


# ---------------------------------------------------------------- the whole

FORMS = {"norm": (_prepare_norm, _own_norm, _plain_norm, _exact_norm, _work_norm),
         "linear8": (_prepare_linear, _own_linear, _plain_linear, _exact_linear, _work_linear),
         "scan": (_prepare_scan, _own_scan, _plain_scan, _exact_scan, _work_scan),
         "adamw": (_prepare_adamw, _own_adamw, _plain_adamw, _exact_adamw, _work_adamw)}


def _form(case, which):
    return FORMS[case["kind"].split("_")[0]][which]


def prepare(case, seed):
    state = {"case": dict(case)}
    _form(case, 0)(case, torch.Generator(device="cuda").manual_seed(int(seed)), state)
    return state


def run(state):
    case = state["case"]
    return _form(case, 1 if own else 2)(case, state)


def exact(case, seed):
    global own
    before, own = own, False  # (its inputs need none of the repository's code)
    try:
        state = prepare(case, seed)
    finally:
        own = before
    return _form(case, 3)(case, state)


def work(case):
    return _form(case, 4)(case)
