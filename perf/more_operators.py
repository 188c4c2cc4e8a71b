"""The operators of a recurrent model that answers with tokens, as they are called, beside their plain forms.

  delta      the gated delta rule S_t = a_t S_{t-1} + k_t u_t^T, u_t = b_t (v_t - a_t S_{t-1}^T k_t), o_t = scale S_t^T q_t over time
             that P workers share, its adjoint, and the step of single tokens
  logprob    log probabilities of given tokens under logits whose vocabulary P workers share, the entropy, the top alternatives;
             and its adjoint
  distill    divergence of such logits from a teacher's top logits, and its gradient

A case is a flat dict.  listed() names twelve, draw() gives more of the same ranges, exact() computes what run() returns
in 64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases

def _delta(dtype, n_b, steps, n_h, n_hk, d_k, d_v, parts, back=False, ragged=False, decay=True, start=True, **name):
    return dict(kind="delta_bwd" if back else "delta_fwd", dtype=dtype, n_b=n_b, steps=steps, n_h=n_h, n_hk=n_hk, d_k=d_k, d_v=d_v,
                parts=parts, ragged=ragged, decay=decay, start=start, **name)


def _step(dtype, rows, n_h, n_hk, d_k, d_v, slots, idle=False, **name):
    return dict(kind="delta_step", dtype=dtype, rows=rows, n_h=n_h, n_hk=n_hk, d_k=d_k, d_v=d_v, slots=slots, idle=idle, **name)


def _logprob(dtype, rows, n_v, parts, n_top=0, entropy=True, back=False, ragged=False, temperature=1.0, **name):
    return dict(kind="logprob_bwd" if back else "logprob_fwd", dtype=dtype, rows=rows, n_v=n_v, parts=parts, n_top=n_top, entropy=entropy,
                ragged=ragged, temperature=temperature, **name)


def _distill(dtype, rows, n_v, parts, n_top, ragged=False, temperature=1.0, **name):
    return dict(kind="distill", dtype=dtype, rows=rows, n_v=n_v, parts=parts, n_top=n_top, ragged=ragged, temperature=temperature, **name)


def listed():
    return [
        # decoding: one token of four sequences, 16 heads, queries and keys shared by two of them
        _step("bf16", 4, 16, 8, 128, 128, 16, name="delta_token"),
        # decoding a batch: 64 sequences whose states lie in a pool of slots, some rows idle
        _step("bf16", 64, 32, 16, 128, 128, 80, idle=True, name="delta_batch"),
        # a long prompt on four time workers: few chains, time is the long axis
        _delta("bf16", 1, 8192, 32, 16, 128, 128, 4, name="delta_prompt"),
        # a ragged batch in 32 bits (one sequence is empty), sizes that nothing divides
        _delta("f32", 5, 1001, 6, 3, 96, 72, 3, ragged=True, name="delta_ragged"),
        # a training step's adjoint on two time workers
        _delta("bf16", 4, 2048, 16, 16, 128, 128, 2, back=True, name="delta_bwd"),
        # the same for a ragged batch in 32 bits, each key's head shared by three, three time workers
        _delta("f32", 3, 515, 6, 2, 64, 80, 3, back=True, ragged=True, name="delta_bwd_ragged"),
        # decoding: log probabilities of eight sampled tokens, the entropy and 20 alternatives
        _logprob("bf16", 8, 65536, 1, 20, name="logprob_token"),
        # the likelihood and entropy of a batch of answers, the vocabulary on four workers
        _logprob("bf16", 8192, 32000, 4, ragged=True, name="logprob_rows"),
        # scoring prompts: five alternatives for each of 2048 tokens, a wide vocabulary on eight workers
        _logprob("bf16", 2048, 131072, 8, 5, entropy=False, temperature=0.7, name="logprob_top"),
        # the adjoint with an odd vocabulary on three workers, gradients of the entropy among them
        _logprob("f32", 1003, 50001, 3, back=True, ragged=True, name="logprob_bwd_odd"),
        # a training step's loss and gradient against 64 teacher logits for each of 4096 tokens; the most bytes
        _distill("bf16", 4096, 131072, 2, 64, ragged=True, temperature=2.0, name="distill_wide"),
        # a small batch with an odd vocabulary in 32 bits
        _distill("f32", 37, 10007, 3, 17, ragged=True, name="distill_odd"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["delta_fwd", "delta_fwd", "delta_bwd", "delta_bwd", "delta_step", "logprob_fwd", "logprob_fwd", "logprob_bwd", "distill"])
    dtype = rng.choice(["f32", "bf16"])
    while True:
        if kind.startswith("delta"):
            n_hk, each = rng.choice([1, 2, 3, 4, 8, 16]), rng.choice([1, 1, 2, 4])
            d_k, d_v = (rng.choice([64, 128]) if rng.random() < 0.6 else _log(rng, 16, 128) for _ in range(2))
            size = n_hk * each * d_k * d_v
            if kind == "delta_step":
                rows = _log(rng, 1, 256)
                if rows * size <= 1 << 25:
                    return _step(dtype, rows, n_hk * each, n_hk, d_k, d_v, rows + rng.randrange(64), rng.random() < 0.5)
                continue
            n_b, steps, parts = _log(rng, 1, 16), _log(rng, 1, 16384), rng.choice([1, 1, 2, 3, 4])
            if n_b * steps * size <= (1 << 31 if kind == "delta_bwd" else 1 << 32) and steps >= parts and (dtype == "bf16" or n_b * steps * size <= 1 << 30):
                return _delta(dtype, n_b, steps, n_hk * each, n_hk, d_k, d_v, parts, kind == "delta_bwd", rng.random() < 0.5,
                              rng.random() < 0.8, rng.random() < 0.5)
        else:
            rows, n_v, parts = _log(rng, 1, 16384), _log(rng, 500, 200000), rng.choice([1, 1, 2, 3, 4, 8])
            n_v = n_v if rng.random() < 0.5 else max(512, n_v // 256 * 256)
            if rows * n_v > (1 << 28 if dtype == "bf16" else 1 << 27):
                continue
            temperature, ragged = rng.choice([1.0, 1.0, 0.7, 2.0]), rng.random() < 0.5
            if kind == "distill":
                return _distill(dtype, rows, n_v, parts, _log(rng, 1, 256), ragged, temperature)
            if kind == "logprob_bwd":
                return _logprob(dtype, rows, n_v, parts, 0, rng.random() < 0.5, True, ragged, temperature)
            n_top = 0 if rng.random() < 0.3 else _log(rng, 1, 64)
            return _logprob(dtype, rows, n_v, parts, n_top, rng.random() < 0.5, False, ragged, temperature)


# ---------------------------------------------------------------- pieces

def _parts(n, parts):
    return [n // parts + (r < n % parts) for r in range(parts)]


def _cut(x, parts, dim):
    return [t.contiguous() for t in x.split(_parts(x.shape[dim], parts), dim)]


def _rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device="cuda")


# ---------------------------------------------------------------- delta

def _prepare_delta(c, gen, s):
    t, n_h, n_hk, d_k, d_v = TYPES[c["dtype"]], c["n_h"], c["n_hk"], c["d_k"], c["d_v"]
    step = c["kind"] == "delta_step"
    lead = (c["rows"],) if step else (c["n_b"], c["steps"])
    unit = lambda v: v / v.square().sum(-1, keepdim=True).add(1e-6).sqrt()  # noqa: E731
    q, k, v = unit(_rand(gen, *lead, n_hk, d_k)).to(t), unit(_rand(gen, *lead, n_hk, d_k)).to(t), _rand(gen, *lead, n_h, d_v).to(t)
    pace = torch.exp(7 * _uniform(gen, n_h) - 6)  # a head forgets within a few steps, or within hundreds
    g = -pace * torch.nn.functional.softplus(_rand(gen, *lead, n_h)) if c.get("decay", True) else None
    beta = torch.sigmoid(_rand(gen, *lead, n_h))
    s["scale"] = d_k ** -0.5
    if step:
        s.update(q=q, k=k, v=v, g=g, beta=beta, o=torch.empty_like(v))
        s["state"] = 0.3 * _rand(gen, c["slots"], n_h, d_k, d_v)
        s["slots"] = torch.randperm(c["slots"], generator=gen, device="cuda")[:c["rows"]].to(torch.int32)
        if c["idle"]:
            s["slots"] = torch.where(_uniform(gen, c["rows"]) < 0.1, -1, s["slots"]).to(torch.int32)
        return
    P = c["parts"]
    cut = lambda x: None if x is None else _cut(x, P, 1)  # noqa: E731
    s.update(q=cut(q), k=cut(k), v=cut(v), g=cut(g), beta=cut(beta))
    s["h0"] = 0.3 * _rand(gen, c["n_b"], n_h, d_k, d_v) if c["start"] else None
    s["lengths"] = None
    if c["ragged"]:
        lengths = torch.randint(0, c["steps"] + 1, (c["n_b"],), generator=gen, device="cuda", dtype=torch.int32)
        lengths[-1] = 0 if c["n_b"] > 2 else c["steps"]
        s["lengths"] = lengths
    like = lambda xs: None if xs is None else [torch.empty_like(x) for x in xs]  # noqa: E731
    if c["kind"] == "delta_fwd":
        s["o"], s["hT"] = like(s["v"]), torch.empty(c["n_b"], n_h, d_k, d_v, device="cuda")
    else:
        s["do"] = cut((1e-3 * _rand(gen, *lead, n_h, d_v)).to(t))
        s["dhT"] = 1e-3 * _rand(gen, c["n_b"], n_h, d_k, d_v)
        for name in ("q", "k", "v", "g", "beta"):
            s["d" + name] = like(s[name])
        s["dh0"] = None if s["h0"] is None else torch.empty_like(s["h0"])
    if own:
        import paper_2006_03108_amd as dd
        s["plan"] = dd.distdl_delta_plan_create(c["n_b"], c["steps"], n_h, n_hk, d_k, d_v, P, s["scale"], t)


def _own_delta(c, s):
    import paper_2006_03108_amd as dd
    if c["kind"] == "delta_step":
        dd.distdl_delta_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["state"], s["slots"], s["o"], s["scale"])
        return {"o": s["o"], "state": s["state"]}
    if c["kind"] == "delta_fwd":
        dd.distdl_delta_fwd(s["plan"], s["q"], s["k"], s["v"], s["g"], s["beta"], s["h0"], s["lengths"], s["o"], s["hT"])
        return {"o": s["o"], "hT": s["hT"]}
    dd.distdl_delta_bwd(s["plan"], s["q"], s["k"], s["v"], s["g"], s["beta"], s["h0"], s["lengths"], s["do"], s["dhT"],
                        s["dq"], s["dk"], s["dv"], s["dg"], s["dbeta"], s["dh0"])
    return {n: s[n] for n in ("dq", "dk", "dv", "dg", "dbeta", "dh0")}


def _unit_inverse(a):
    """(1 + a)^-1 of strictly lower [..., n, n], n a power of two: blocks along the diagonal, two become one."""
    n, inv = a.shape[-1], torch.ones_like(a[..., :1, None])
    size = 1
    while size < n:
        both = a.unflatten(-1, (-1, 2 * size)).unflatten(-3, (-1, 2 * size)).diagonal(dim1=-4, dim2=-2).movedim(-1, -3)
        top, bottom = inv[..., 0::2, :, :], inv[..., 1::2, :, :]
        low = -(bottom @ (both[..., size:, :size] @ top))
        inv = torch.cat([torch.cat([top, torch.zeros_like(top)], -1), torch.cat([low, bottom], -1)], -2)
        size *= 2
    return inv[..., 0, :, :]


def _chunked(q, k, v, g, beta, state, scale):
    """(o, last state) from fp32 [n, heads, steps, ...], in chunks of 64 steps: what the steps of a chunk do to each other is one product."""
    n, n_h, T, d_k = q.shape
    size = 64 if T > 32 else 1 << max(0, T - 1).bit_length()
    fold = lambda x: torch.nn.functional.pad(x, (0, 0, 0, -T % size)).unflatten(2, (-1, size))  # noqa: E731
    q, k, v, beta = fold(q), fold(k), fold(v), fold(beta[..., None])
    total = fold(g[..., None])[..., 0].double().cumsum(-1)
    low = torch.ones(size, size, dtype=torch.bool, device=q.device).tril()
    decay = torch.where(low, total[..., :, None] - total[..., None, :], -torch.inf).exp().float()
    total = total.float()[..., None]
    inner = _unit_inverse((beta * decay * (k @ k.transpose(-1, -2))).tril(-1))
    among = scale * decay * (q @ k.transpose(-1, -2))
    since, until, whole = total.exp(), (total[..., -1:, :] - total).exp(), total[..., -1:, :].exp()
    out = []
    for i in range(q.shape[2]):
        u = inner[:, :, i] @ (beta[:, :, i] * (v[:, :, i] - since[:, :, i] * (k[:, :, i] @ state)))
        out.append(scale * since[:, :, i] * (q[:, :, i] @ state) + among[:, :, i] @ u)
        state = whole[:, :, i] * state + k[:, :, i].transpose(-1, -2) @ (until[:, :, i] * u)
    return torch.stack(out, 2).flatten(2, 3)[:, :, :T], state


def _plain_delta(c, s):
    t, each = TYPES[c["dtype"]], c["n_h"] // c["n_hk"]
    if c["kind"] == "delta_step":
        live, at = s["slots"] >= 0, s["slots"].long().clamp(min=0)
        q, k = (s[n].float().repeat_interleave(each, 1) for n in ("q", "k"))
        h = s["state"][at]
        decayed = h * s["g"].exp()[:, :, None, None]
        u = s["beta"][:, :, None] * (s["v"].float() - (decayed * k[..., None]).sum(2))
        new = decayed + k[..., None] * u[:, :, None]
        o = s["scale"] * (new * q[..., None]).sum(2)
        s["state"].index_add_(0, at, torch.where(live[:, None, None, None], new - h, 0.0))
        return {"o": torch.where(live[:, None, None], o, 0.0).to(t), "state": s["state"]}
    P, T = c["parts"], c["steps"]
    names = [n for n in ("q", "k", "v", "g", "beta") if s[n] is not None]
    leaves = {n: torch.cat(s[n], 1).float() for n in names}
    h0 = torch.zeros(c["n_b"], c["n_h"], c["d_k"], c["d_v"], device="cuda") if s["h0"] is None else s["h0"].clone()
    back = c["kind"] == "delta_bwd"
    for x in [*leaves.values(), h0] if back else []:
        x.requires_grad_()
    inside = None if s["lengths"] is None else torch.arange(T, device="cuda")[None] < s["lengths"][:, None]
    with torch.set_grad_enabled(back):
        x = {n: leaves[n] if inside is None else torch.where(inside.view(*inside.shape, *[1] * (leaves[n].dim() - 2)), leaves[n], 0.0) for n in names}
        q, k = (x[n].repeat_interleave(each, 2).transpose(1, 2) for n in ("q", "k"))
        g = x["g"] if "g" in x else torch.zeros_like(x["beta"])
        o, hT = _chunked(q, k, x["v"].transpose(1, 2), g.transpose(1, 2), x["beta"].transpose(1, 2), h0, s["scale"])
        o = o.transpose(1, 2)
    if not back:
        return {"o": _cut(o.to(t), P, 1), "hT": hT}
    do = torch.cat(s["do"], 1).float()
    do = do if inside is None else torch.where(inside[:, :, None, None], do, 0.0)
    grads = torch.autograd.grad([o, hT], [*leaves.values(), h0], [do, s["dhT"]])
    out = {"d" + n: _cut(v.to(s[n][0].dtype), P, 1) for n, v in zip(names, grads)}
    return {**out, "dg": out.get("dg"), "dh0": None if s["h0"] is None else grads[-1]}


def _exact_delta(c, s):
    """Step by step."""
    each = c["n_h"] // c["n_hk"]
    if c["kind"] == "delta_step":
        o, state = torch.zeros_like(s["v"], dtype=torch.float64), s["state"].double()
        for row, slot in enumerate(s["slots"].tolist()):
            if slot < 0:
                continue
            q, k, v, b = (s[n][row].double() for n in ("q", "k", "v", "beta"))
            a = s["g"][row].double().exp()
            q, k = q.repeat_interleave(each, 0), k.repeat_interleave(each, 0)
            h = state[slot] * a[:, None, None]
            h = h + torch.einsum("hk,hv->hkv", k, b[:, None] * (v - torch.einsum("hkv,hk->hv", h, k)))
            state[slot], o[row] = h, s["scale"] * torch.einsum("hkv,hk->hv", h, q)
        return {"o": o, "state": state}
    P, T, scale = c["parts"], c["steps"], s["scale"]
    q, k, v, beta = (torch.cat(s[n], 1).double() for n in ("q", "k", "v", "beta"))
    q, k = q.repeat_interleave(each, 2), k.repeat_interleave(each, 2)
    a = torch.ones_like(beta) if s["g"] is None else torch.cat(s["g"], 1).double().exp()
    if s["lengths"] is not None:  # steps behind the end do nothing: their factor is 1, their key 0
        inside = torch.arange(T, device="cuda")[None] < s["lengths"][:, None]
        q, k, v = (torch.where(inside[:, :, None, None], x, 0.0) for x in (q, k, v))
        a, beta = torch.where(inside[:, :, None], a, 1.0), torch.where(inside[:, :, None], beta, 0.0)
    h = torch.zeros(c["n_b"], c["n_h"], c["d_k"], c["d_v"], dtype=torch.float64, device="cuda") if s["h0"] is None else s["h0"].double()
    times = lambda m, x: (m @ x[..., None])[..., 0]  # noqa: E731
    turned = lambda m, x: (x[..., None, :] @ m)[..., 0, :]  # noqa: E731

    def step(h, i):
        """(state before, r, state after)"""
        before = h * a[:, i, :, None, None]
        r = v[:, i] - turned(before, k[:, i])
        return before, r, torch.addcmul(before, k[:, i, :, :, None], (beta[:, i, :, None] * r)[..., None, :])

    if c["kind"] == "delta_fwd":
        o = torch.empty_like(v)
        for i in range(T):
            h = step(h, i)[2]
            o[:, i] = scale * turned(h, q[:, i])
        return {"o": _cut(o, P, 1), "hT": h}
    run, marks = 64, []
    for i in range(T):  # a state for each 64 steps; those between are made again
        if i % run == 0:
            marks.append(h)
        h = step(h, i)[2]
    do = torch.cat(s["do"], 1).double()
    if s["lengths"] is not None:
        do = torch.where(inside[:, :, None, None], do, 0.0)
    dq, dk, dv, dg, dbeta = (torch.empty_like(x) for x in (q, k, v, a, beta))
    dh = s["dhT"].double()
    for first in range((T - 1) // run * run, -1, -run):
        states = [marks.pop()]
        for i in range(first, min(first + run, T)):
            states.append(step(states[-1], i)[2])
        for i in range(min(first + run, T) - 1, first - 1, -1):
            after, (before, r, _) = states[i - first + 1], step(states[i - first], i)
            dq[:, i] = scale * times(after, do[:, i])
            dh = torch.addcmul(dh, q[:, i, :, :, None], do[:, i, :, None, :], value=scale)
            u, du = beta[:, i, :, None] * r, turned(dh, k[:, i])
            dr = beta[:, i, :, None] * du
            dv[:, i], dbeta[:, i] = dr, (du * r).sum(-1)
            dk[:, i] = times(dh, u) - times(before, dr)
            dh = torch.addcmul(dh, k[:, i, :, :, None], dr[..., None, :], value=-1)
            dg[:, i] = (dh * before).sum((-1, -2))
            dh = dh * a[:, i, :, None, None]
    if s["lengths"] is not None:
        dq, dk, dv = (torch.where(inside[:, :, None, None], x, 0.0) for x in (dq, dk, dv))
        dg, dbeta = (torch.where(inside[:, :, None], x, 0.0) for x in (dg, dbeta))
    shared = lambda x: x.unflatten(2, (-1, each)).sum(3)  # noqa: E731
    return {"dq": _cut(shared(dq), P, 1), "dk": _cut(shared(dk), P, 1), "dv": _cut(dv, P, 1),
            "dg": None if s["g"] is None else _cut(dg, P, 1), "dbeta": _cut(dbeta, P, 1), "dh0": None if s["h0"] is None else dh}


def _work_delta(c):
    size, state = 4 if c["dtype"] == "f32" else 2, c["n_h"] * c["d_k"] * c["d_v"]
    token = size * (2 * c["n_hk"] * c["d_k"] + c["n_h"] * c["d_v"]) + 4 * c["n_h"] * (1 + c.get("decay", True))  # q, k, v, g, beta
    if c["kind"] == "delta_step":
        rows = c["rows"] * (0.9 if c["idle"] else 1.0)
        return {"bytes": rows * (8 * state + token) + c["rows"] * size * c["n_h"] * c["d_v"], "flops": 7 * rows * state}
    tokens, share = c["n_b"] * c["steps"], 0.5 if c["ragged"] else 1.0  # steps behind a sequence's end are written, not read
    out = size * c["n_h"] * c["d_v"]
    ends = 4 * c["n_b"] * state * (1 + c["start"])
    if c["kind"] == "delta_fwd":
        return {"bytes": tokens * (share * token + out) + ends, "flops": 7 * share * tokens * state}
    return {"bytes": tokens * (share * (token + out) + token) + ends + 4 * c["n_b"] * state * c["start"], "flops": 20 * share * tokens * state}


# ---------------------------------------------------------------- logprob

def _prepare_logits(c, gen, s):
    """Logits as a last layer leaves them: the vocabulary is filled up to its size with entries that no answer has."""
    rows, n_v, t = c["rows"], c["n_v"], TYPES[c["dtype"]]
    real = s["real"] = n_v - n_v // 100
    x = torch.empty(rows, n_v, dtype=t, device="cuda")
    for r in range(0, rows, 1024):
        part = x[r:r + 1024]
        part.copy_(2.5 * _rand(gen, *part.shape))
    x[:, real:] = -torch.inf
    s["x"] = _cut(x, c["parts"], 1)
    return x


def _prepare_logprob(c, gen, s):
    rows = c["rows"]
    x = _prepare_logits(c, gen, s)
    target = torch.randint(0, s["real"], (rows,), generator=gen, device="cuda")
    # most tokens are likely ones: the largest logit of some that are picked at random
    some = torch.randint(0, s["real"], (rows, 64), generator=gen, device="cuda")
    likely = some.gather(1, x.gather(1, some).argmax(1, keepdim=True))[:, 0]
    target = torch.where(_uniform(gen, rows) < 0.8, likely, target)
    if c["ragged"]:  # rows of padding
        target = torch.where(_uniform(gen, rows) < 0.1, -1, target)
    s["target"] = target.to(torch.int32)
    new = lambda *shape, kind=torch.float32: torch.empty(*shape, dtype=kind, device="cuda")  # noqa: E731
    if c["kind"] == "logprob_fwd":
        s["logp"], s["lse"], s["entropy"] = new(rows), new(rows), new(rows) if c["entropy"] else None
        s["ids"], s["top"] = (new(rows, c["n_top"], kind=torch.int32), new(rows, c["n_top"])) if c["n_top"] else (None, None)
    else:
        s["lse"], s["entropy"] = new(rows), new(rows) if c["entropy"] else None
        for r in range(0, rows, 512):
            z = x[r:r + 512, :s["real"]].double() / c["temperature"]
            lse = z.logsumexp(1)
            s["lse"][r:r + 512] = lse
            if c["entropy"]:
                s["entropy"][r:r + 512] = lse - ((z - lse[:, None]).exp() * z).sum(1)
        s["dlogp"] = -(1 + 0.3 * _rand(gen, rows)) / rows  # an answer's weight, over the batch
        s["dentropy"] = torch.full((rows,), -0.01 / rows, device="cuda") if c["entropy"] else None
        s["dx"] = [torch.empty_like(v) for v in s["x"]]
    if own:
        import paper_2006_03108_amd as dd
        s["plan"] = dd.distdl_logits_plan_create(rows, c["n_v"], c["parts"], TYPES[c["dtype"]])


def _own_logprob(c, s):
    import paper_2006_03108_amd as dd
    if c["kind"] == "logprob_fwd":
        dd.distdl_logprob_fwd(s["plan"], s["x"], s["target"], s["logp"], s["lse"], s["entropy"], s["ids"], s["top"], c["temperature"])
        return {k: s[k] for k in ("logp", "lse", "entropy", "ids", "top")}
    dd.distdl_logprob_bwd(s["plan"], s["x"], s["target"], s["lse"], s["entropy"], s["dlogp"], s["dentropy"], s["dx"], c["temperature"])
    return {"dx": s["dx"]}


def _plain_logprob(c, s):
    z = torch.cat(s["x"], 1).float() / c["temperature"]
    live, at = s["target"] >= 0, s["target"].long().clamp(min=0)[:, None]
    if c["kind"] == "logprob_fwd":
        most = z.amax(1, keepdim=True)
        e = (z - most).exp()
        total = e.sum(1)
        lse = most[:, 0] + total.log()
        out = {"logp": torch.where(live, z.gather(1, at)[:, 0] - lse, 0.0), "lse": lse, "entropy": None, "ids": None, "top": None}
        if c["entropy"]:
            out["entropy"] = total.log() - torch.where(e > 0, e * (z - most), 0.0).sum(1) / total
        if c["n_top"]:
            value, order = z.sort(dim=1, descending=True, stable=True)
            out["ids"], out["top"] = order[:, :c["n_top"]].to(torch.int32), value[:, :c["n_top"]] - lse[:, None]
        return out
    log_p = z - s["lse"][:, None]
    p = log_p.exp()
    weight = torch.where(live, s["dlogp"], 0.0)
    dz = -weight[:, None] * p
    dz.scatter_add_(1, at, weight[:, None])
    if c["entropy"]:
        dz -= s["dentropy"][:, None] * torch.where(p > 0, p * (log_p + s["entropy"][:, None]), 0.0)
    return {"dx": _cut((dz / c["temperature"]).to(TYPES[c["dtype"]]), c["parts"], 1)}


def _exact_logprob(c, s):
    """From the entries that an answer can have; a thousand rows at a time."""
    out = {n: [] for n in ("logp", "lse", "entropy", "ids", "top", "dx")}
    for r in range(0, c["rows"], 1024):
        rows = slice(r, r + 1024)
        z = torch.cat([v[rows] for v in s["x"]], 1)[:, :s["real"]].double() / c["temperature"]
        target, each = s["target"][rows].long(), torch.arange(z.shape[0], device="cuda")
        if c["kind"] == "logprob_fwd":
            lse = torch.logsumexp(z, 1)
            out["lse"].append(lse)
            out["logp"].append(torch.where(target < 0, 0.0, z[each, target] - lse))
            if c["entropy"]:
                log_p = z - lse[:, None]
                out["entropy"].append(-(log_p.exp() * log_p).sum(1))
            for _ in range(c["n_top"]):  # the largest, at its first place; it is taken out for the next
                value = z.amax(1)
                place = torch.where(z == value[:, None], torch.arange(z.shape[1], device="cuda"), z.shape[1]).amin(1)
                out["ids"].append(place.to(torch.int32))
                out["top"].append(value - lse)
                z[each, place] = -torch.inf
            continue
        log_p = z - s["lse"][rows].double()[:, None]
        p = log_p.exp()
        weight = torch.where(target < 0, 0.0, s["dlogp"][rows].double())
        dz = torch.zeros(z.shape[0], c["n_v"], dtype=torch.float64, device="cuda")
        dz[:, :s["real"]] = -p * weight[:, None]
        if c["entropy"]:
            dz[:, :s["real"]] -= s["dentropy"][rows].double()[:, None] * p * (log_p + s["entropy"][rows].double()[:, None])
        dz[each, target.clamp(min=0)] += weight
        out["dx"].append(dz / c["temperature"])
    if c["kind"] == "logprob_bwd":
        return {"dx": _cut(torch.cat(out["dx"]), c["parts"], 1)}
    of = lambda n: torch.cat(out[n]) if out[n] else None  # noqa: E731
    k = c["n_top"]
    top = {n: torch.cat([torch.stack(out[n][i:i + k], 1) for i in range(0, len(out[n]), k)]) if k else None for n in ("ids", "top")}
    return {"logp": of("logp"), "lse": of("lse"), "entropy": of("entropy"), **top}


def _work_logprob(c):
    n, size = c["rows"] * c["n_v"], 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "logprob_fwd":
        return {"bytes": n * size + c["rows"] * (12 + 4 * c["entropy"] + 8 * c["n_top"]), "flops": (6 if c["entropy"] else 4) * n}
    return {"bytes": 2 * n * size + c["rows"] * (12 + 8 * c["entropy"]), "flops": (8 if c["entropy"] else 4) * n}


# ---------------------------------------------------------------- distill

def _prepare_distill(c, gen, s):
    rows, k = c["rows"], min(c["n_top"], c["n_v"] // 2)
    x = _prepare_logits(c, gen, s)
    ids, teacher = [], []
    for r in range(0, rows, 512):  # a teacher that the student has learnt something of
        z = x[r:r + 512, :s["real"]].float()
        best = (0.8 * z + 1.5 * _rand(gen, *z.shape)).topk(k)
        ids.append(best.indices)
        teacher.append(best.values)
    s["ids"], s["teacher"] = torch.cat(ids).to(torch.int32), torch.cat(teacher)
    s["weight"] = torch.full((rows,), 1 / rows, device="cuda")
    if c["ragged"]:  # a teacher may have stored fewer, and rows of padding have none
        kept = torch.randint(1, k + 1, (rows, 1), generator=gen, device="cuda")
        kept = torch.where(_uniform(gen, rows, 1) < 0.5, kept, k)
        kept = torch.where(_uniform(gen, rows, 1) < 0.1, 0, kept)
        s["ids"] = torch.where(torch.arange(k, device="cuda")[None] < kept, s["ids"], -1).to(torch.int32)
        s["weight"] = torch.where(kept[:, 0] > 0, s["weight"], 0.0)
    s["loss"], s["dx"] = torch.empty(rows, device="cuda"), [torch.empty_like(v) for v in s["x"]]
    if own:
        import paper_2006_03108_amd as dd
        s["plan"] = dd.distdl_logits_plan_create(rows, c["n_v"], c["parts"], TYPES[c["dtype"]])


def _own_distill(c, s):
    import paper_2006_03108_amd as dd
    dd.distdl_distill_fwd_bwd(s["plan"], s["x"], s["ids"], s["teacher"], s["weight"], s["loss"], s["dx"], c["temperature"])
    return {"loss": s["loss"], "dx": s["dx"]}


def _plain_distill(c, s):
    z = torch.cat(s["x"], 1).float() / c["temperature"]
    most = z.amax(1, keepdim=True)
    e = (z - most).exp()
    total = e.sum(1, keepdim=True)
    stored, at = s["ids"] >= 0, s["ids"].long().clamp(min=0)
    any_ = stored.any(1)
    t = torch.where(stored, s["teacher"] / c["temperature"], -torch.inf)
    t = t - torch.where(any_, t.amax(1), 0.0)[:, None]
    mass = torch.where(any_, t.exp().sum(1), 1.0)[:, None]
    p = t.exp() / mass
    loss = torch.where(p > 0, p * (t - mass.log() - (z.gather(1, at) - most - total.log())), 0.0).sum(1)
    weight = torch.where(any_, s["weight"], 0.0)[:, None] / c["temperature"]
    dz = weight * (e / total)
    dz.scatter_add_(1, at, -weight * p)
    return {"loss": loss, "dx": _cut(dz.to(TYPES[c["dtype"]]), c["parts"], 1)}


def _exact_distill(c, s):
    loss, grads = [], []
    for r in range(0, c["rows"], 1024):
        rows = slice(r, r + 1024)
        z = torch.cat([v[rows] for v in s["x"]], 1)[:, :s["real"]].double() / c["temperature"]
        log_q = z - torch.logsumexp(z, 1, keepdim=True)
        kept = (s["ids"][rows] >= 0).sum(1, keepdim=True)  # they come first
        inside = torch.arange(s["ids"].shape[1], device="cuda")[None] < kept
        log_p = torch.log_softmax(torch.where(inside, s["teacher"][rows].double() / c["temperature"], -1e9), 1)
        p = torch.where(inside, log_p.exp(), 0.0)
        at = torch.where(inside, s["ids"][rows].long(), 0)
        loss.append((p * (log_p - log_q.gather(1, at))).sum(1))
        weight = torch.where(kept > 0, s["weight"][rows].double()[:, None], 0.0)
        dz = torch.zeros(z.shape[0], c["n_v"], dtype=torch.float64, device="cuda")
        dz[:, :s["real"]] = log_q.exp()
        dz.scatter_add_(1, at, -p)
        grads.append(dz * weight / c["temperature"])
    return {"loss": torch.cat(loss), "dx": _cut(torch.cat(grads), c["parts"], 1)}


def _work_distill(c):
    n, size = c["rows"] * c["n_v"], 4 if c["dtype"] == "f32" else 2
    return {"bytes": 2 * n * size + c["rows"] * (8 + 8 * c["n_top"]), "flops": 6 * n}


# ---------------------------------------------------------------- the whole

FORMS = {"delta": (_prepare_delta, _own_delta, _plain_delta, _exact_delta, _work_delta),
         "logprob": (_prepare_logprob, _own_logprob, _plain_logprob, _exact_logprob, _work_logprob),
         "distill": (_prepare_distill, _own_distill, _plain_distill, _exact_distill, _work_distill)}


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
