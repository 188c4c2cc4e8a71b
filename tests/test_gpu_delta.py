"""The gated delta rule on the GPU against the oracle, step by step in fp64.

Tolerances, in the 2-norm of each output.  u = 2^-24.  Keys have unit length, beta and the factors are at most 1, so a step is no longer than its input
and what an earlier chunk's rounding adds does not grow.  A chunk is four products one behind the other whose sums have up to 128 terms of 24 bits,
each of them rounded like a sum of 128 terms, sqrt(128) u of its size: 48 u for a chunk of 32 steps, and one more for what is left: 48 u (1 + T / 32).
bf16 outputs are rounded once more, by up to 2^-8, and what they alone depend on has 16 bits (2^-15 in a product of two): 2^-8 + 2^-13.

What is rounded is a sum's terms.  Those of an output, and of the gradients of a step, are products of numbers of size one with `scale` (o = scale (a q h0 +
(q k) beta (v - a k h0)) for one step of one number), and a sum of few of them may cancel: 1.8e-9 off, 0.03 u, is 62 u of an o of 4.9e-4.  So the size that
the limit is of is no less than scale for each number of those outputs."""
import numpy as np
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from oracle import tokens

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def limit(t, T):
    return 2.0 ** -8 + 2.0 ** -13 if t.dtype == BF16 else 48 * U * (1 + T / 32)


def near(got, want, tol, what, least=0.0):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    assert np.isfinite(got).all(), what
    off, size = np.linalg.norm((got - want).ravel()), max(np.linalg.norm(want.ravel()), least * np.sqrt(want.size))
    assert off <= tol * size + 1e-30, f"{what}: {off / max(size, 1e-300):.3e} > {tol:.3e}"


def cut(x, parts):
    T = x.shape[1]
    return [t.contiguous().cuda() for t in x.split([T // parts + (r < T % parts) for r in range(parts)], 1)]


def make(n_b, T, n_h, n_hk, d_k, d_v, dtype, seed=0, pace=None, decay=True):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    q, k, v = unit(r(n_b, T, n_hk, d_k)).to(dtype), unit(r(n_b, T, n_hk, d_k)).to(dtype), r(n_b, T, n_h, d_v).to(dtype)
    if dtype == BF16:  # (rounding may make a key longer than 1)
        k = (k * 0.995).to(BF16)
    pace = torch.exp(6 * torch.rand(n_h, generator=g) - 5) if pace is None else torch.full((n_h,), pace)
    gate = -pace * torch.nn.functional.softplus(r(n_b, T, n_h)) if decay else torch.zeros(n_b, T, n_h)
    return dict(q=q, k=k, v=v, g=gate, beta=torch.sigmoid(r(n_b, T, n_h)), h0=r(n_b, n_h, d_k, d_v), do=r(n_b, T, n_h, d_v).to(dtype),
                dhT=0.1 * r(n_b, n_h, d_k, d_v))


def lengths_of(n_b, T, seed=0):
    lengths = torch.randint(0, T + 1, (n_b,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    lengths[0] = T
    if n_b > 2:
        lengths[2] = 0
    return lengths


def numpy_of(x, start=True):
    out = {n: t.double().numpy() for n, t in x.items()}
    if not start:
        out["h0"] = np.zeros_like(out["h0"])
    return out


def run(x, lengths, parts, scale, decay=True, start=True, back=True, out=None):
    n_b, T, n_h, d_v = x["v"].shape
    n_hk, d_k = x["q"].shape[2:]
    plan = dd.distdl_delta_plan_create(n_b, T, n_h, n_hk, d_k, d_v, parts, scale, x["v"].dtype)
    c = {n: cut(x[n], parts) for n in ("q", "k", "v", "g", "beta", "do")}
    g, h0 = c["g"] if decay else None, x["h0"].cuda() if start else None
    lengths = None if lengths is None else lengths.cuda()
    like = lambda ts: [torch.full_like(t, 7.0) for t in ts]  # noqa: E731
    o, hT = like(c["v"]), torch.full(x["h0"].shape, 7.0, device="cuda")
    dd.distdl_delta_fwd(plan, c["q"], c["k"], c["v"], g, c["beta"], h0, lengths, o, hT)
    got = dict(o=torch.cat(o, 1), hT=hT)
    if back:
        d = {n: like(c[n]) for n in ("q", "k", "v", "g", "beta")}
        dh0 = torch.full_like(hT, 7.0) if start else None
        dd.distdl_delta_bwd(plan, c["q"], c["k"], c["v"], g, c["beta"], h0, lengths, c["do"], x["dhT"].cuda(), d["q"], d["k"], d["v"],
                            d["g"] if decay else None, d["beta"], dh0)
        got.update({"d" + n: torch.cat(t, 1) for n, t in d.items() if n != "g" or decay}, **({"dh0": dh0} if start else {}))
    return got


def check(x, lengths, parts, scale=0.3, decay=True, start=True, back=True, factor=1.0):
    got = run(x, lengths, parts, scale, decay, start, back)
    n, T = numpy_of(x, start), x["v"].shape[1]
    ends = np.full(x["v"].shape[0], T) if lengths is None else lengths.numpy().clip(0, T)
    args = (n["q"], n["k"], n["v"], n["g"], n["beta"], n["h0"], ends, scale)
    want = dict(zip(("o", "hT"), tokens.delta_forward(*args)))
    if back:
        want.update(zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), tokens.delta_adjoint(*args, n["do"], n["dhT"])))
    for name, t in got.items():
        near(t, want[name], factor * limit(t, T), name, scale if name in ("o", "dq", "dk", "dv", "dbeta") else 0.0)
    behind = np.arange(T)[None] >= ends[:, None]
    for name in ("o", "dq", "dk", "dv", "dg", "dbeta"):
        if name in got:
            assert (got[name].double().cpu().numpy()[behind] == 0).all(), name
    return got


# n_b, T, n_h, n_hk, d_k, d_v, workers
SIZES = [(1, 1, 1, 1, 1, 1, 1), (2, 3, 2, 1, 5, 7, 2), (1, 31, 2, 2, 16, 16, 1), (1, 32, 1, 1, 64, 32, 1), (2, 33, 3, 1, 33, 17, 3), (1, 64, 2, 1, 128, 128, 1),
         (3, 65, 4, 2, 96, 72, 2), (2, 150, 2, 2, 65, 40, 3), (1, 200, 6, 3, 128, 130, 4), (1, 40, 1, 1, 20, 300, 20), (2, 129, 4, 4, 64, 64, 2)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_forward(size, dtype):
    require_gpu()
    *shape, parts = size
    x = make(*shape, dtype)
    check(x, lengths_of(shape[0], shape[1]) if shape[0] > 1 else None, parts, back=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_adjoint(size, dtype):
    require_gpu()
    *shape, parts = size
    x = make(*shape, dtype, seed=1)
    check(x, lengths_of(shape[0], shape[1], 1) if shape[0] > 1 else None, parts)


@pytest.mark.parametrize("decay, start", [(False, True), (True, False), (False, False)])
def test_without_decay_or_start(decay, start):
    require_gpu()
    for dtype in (F32, BF16):
        check(make(2, 100, 2, 1, 48, 24, dtype, 2, decay=decay), None, 2, decay=decay, start=start)


def test_many_chains_take_two_tiles_of_columns():
    require_gpu()
    for dtype in (F32, BF16):
        check(make(4, 70, 256, 64, 32, 40, dtype, 3), lengths_of(4, 70, 3), 2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [(33, 70, 6, 2, 24, 20, 2), (65, 40, 4, 2, 100, 40, 1), (2, 70, 140, 1, 20, 16, 1)])
def test_heads_of_many_chunks_and_many_heads_of_few(size, dtype):
    """More chunks of keys than 128, each with several heads, which one workgroup adds up; and few with more heads than there are workgroups for them (the sizes above
    have few of both)."""
    require_gpu()
    n_b, T, n_h, n_hk, d_k, d_v, parts = size
    check(make(n_b, T, n_h, n_hk, d_k, d_v, dtype, seed=5), lengths_of(n_b, T, 5), parts)


def test_lengths_out_of_range_are_cut():
    require_gpu()
    x = make(3, 50, 2, 1, 32, 32, F32, 4)
    check(x, torch.tensor([-5, 1 << 30, 20], dtype=torch.int32), 2)


def test_what_lies_behind_a_sequence_s_end_is_not_read():
    require_gpu()
    for dtype in (F32, BF16):
        x, lengths = make(3, 90, 2, 1, 40, 40, dtype, 5), torch.tensor([90, 33, 0], dtype=torch.int32)
        clean = run(x, lengths, 2, 0.3)
        for i, n in enumerate(lengths.tolist()):
            for name in ("q", "k", "v", "g", "beta", "do"):
                x[name][i, n:] = torch.nan if name != "g" else torch.inf
        for a, b in zip(clean.values(), run(x, lengths, 2, 0.3).values()):
            assert torch.equal(a, b)


def test_factors_of_zero_and_near_it():
    """g of -inf, -1000 and -150 are resets: the state in front has no share.  Small paces keep G exact over a chunk."""
    require_gpu()
    for dtype in (F32, BF16):
        x = make(1, 130, 3, 1, 32, 32, dtype, 6)
        x["g"][0, 5], x["g"][0, 40:44], x["g"][0, 100] = -torch.inf, -1000.0, -150.0
        got = run(x, None, 2, 0.3)
        n = numpy_of(x)
        n["g"] = np.where(n["g"] < -200, -np.inf, n["g"])
        args = (n["q"], n["k"], n["v"], n["g"], n["beta"], n["h0"], np.array([130]), 0.3)
        want = dict(zip(("o", "hT"), tokens.delta_forward(*args)))
        want.update(zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), tokens.delta_adjoint(*args, n["do"], n["dhT"])))
        for name, t in got.items():
            near(t, want[name], limit(t, 130), name)


def test_equal_keys_and_full_updates():
    """All keys alike and beta of 1: T is as far from 1 as it can be, and every step replaces what the key holds."""
    require_gpu()
    for dtype in (F32, BF16):
        x = make(1, 128, 2, 2, 64, 32, dtype, 7, decay=False)
        x["k"] = torch.zeros_like(x["k"])
        x["k"][..., 3] = 1.0
        x["beta"] = torch.ones_like(x["beta"])
        check(x, None, 1, decay=False)


def test_beta_of_zero_and_of_two():
    require_gpu()
    for dtype in (F32, BF16):
        x = make(1, 100, 2, 1, 32, 16, dtype, 8)
        x["beta"][0, ::3] = 0.0
        x["beta"][0, 1::3] = 2.0  # (a reflection; still no longer)
        check(x, None, 2)


def test_shared_keys_add_up_in_order():
    """Gradients of shared keys are the same bits every time, and the sum of those of keys of their own."""
    require_gpu()
    x = make(2, 80, 8, 2, 32, 32, F32, 9)
    a, b = (run(x, None, 2, 0.3) for _ in range(2))
    for name in a:
        assert torch.equal(a[name], b[name]), name
    y = dict(x, q=x["q"].repeat_interleave(4, 2), k=x["k"].repeat_interleave(4, 2))
    own = run(y, None, 2, 0.3)
    for name in ("dq", "dk"):
        near(a[name], own[name].unflatten(2, (2, 4)).double().sum(3).cpu().numpy(), limit(a[name], 80), name)


def test_the_adjoint_of_the_oracle_is_the_derivative():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(2, 5, 1, 3)), rng.normal(size=(2, 5, 1, 3)) * 0.4, rng.normal(size=(2, 5, 2, 2))
    g, beta, h0 = -rng.random(size=(2, 5, 2)), rng.random(size=(2, 5, 2)), rng.normal(size=(2, 2, 3, 2))
    do, dhT, ends = rng.normal(size=v.shape), rng.normal(size=h0.shape), np.array([5, 3])
    ins = [q, k, v, g, beta, h0]

    def value(ins):
        o, hT = tokens.delta_forward(*ins, ends, 0.7)
        return (o * do).sum() + (hT * dhT).sum()
    for i, d in enumerate(tokens.delta_adjoint(*ins, ends, 0.7, do, dhT)):
        for at in np.ndindex(d.shape):
            both = []
            for sign in (1, -1):
                moved = [t.copy() for t in ins]
                moved[i][at] += sign * 1e-5
                both.append(value(moved))
            assert abs((both[0] - both[1]) / 2e-5 - d[at]) < 1e-7


def test_the_kernels_gradient_is_a_difference():
    """Along a random direction of all inputs: <gradient, d> against the oracle's forward values at x + d and x - d."""
    require_gpu()
    x = make(1, 70, 2, 1, 24, 20, F32, 10)
    got, n = run(x, None, 2, 0.5), numpy_of(x)
    rng, names = np.random.default_rng(1), ("q", "k", "v", "g", "beta", "h0")
    d = {m: rng.normal(size=n[m].shape) for m in names}

    def value(step):
        o, hT = tokens.delta_forward(*[n[m] + step * d[m] for m in names], np.array([70]), 0.5)
        return (o * n["do"]).sum() + (hT * n["dhT"]).sum()
    slope = (value(1e-6) - value(-1e-6)) / 2e-6
    mine = sum((got["d" + m].double().cpu().numpy() * d[m]).sum() for m in names)
    size = np.sqrt(sum(np.linalg.norm(got["d" + m].double().cpu().numpy()) ** 2 * np.linalg.norm(d[m]) ** 2 / d[m].size for m in names))
    assert abs(mine - slope) <= 1e-4 * size


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, n_h, n_hk, d_k, d_v", [(1, 1, 1, 1, 1), (3, 2, 1, 5, 7), (4, 4, 2, 128, 128), (2, 3, 3, 96, 72), (5, 2, 2, 64, 33), (2, 2, 1, 128, 260),
                                                      (70, 8, 4, 128, 128), (70, 8, 8, 17, 36)])
def test_step(rows, n_h, n_hk, d_k, d_v, dtype):
    """One product of up to 128 terms each: 2 sqrt(128) u, and bf16's rounding."""
    require_gpu()
    x = make(1, rows, n_h, n_hk, d_k, d_v, dtype, 11)
    pool = torch.randn(rows + 5, n_h, d_k, d_v, generator=torch.Generator().manual_seed(1))
    slots = torch.randperm(rows + 5, generator=torch.Generator().manual_seed(2))[:rows].to(torch.int32)
    if rows > 2:
        slots[1], slots[2] = -1, rows + 5
    q, k, v, g, beta = (x[n][0].contiguous().cuda() for n in ("q", "k", "v", "g", "beta"))
    for with_slots in (True, False):
        for with_gate in (True, False):
            state, o = pool.cuda(), torch.full_like(v, 7.0)
            dd.distdl_delta_step(q, k, v, g if with_gate else None, beta, state, slots.cuda() if with_slots else None, o, 0.25)
            at = slots.long() if with_slots else torch.arange(rows)
            live = ((at >= 0) & (at < rows + 5)).numpy()
            n = {m: x[m][0].double().numpy()[live] for m in ("q", "k", "v", "g", "beta")}
            per = n_h // n_hk
            want_o, want = tokens.delta_step(pool.double().numpy()[at[live]], n["q"].repeat(per, 1), n["k"].repeat(per, 1), n["v"],
                                             np.exp(n["g"] * with_gate), n["beta"], 0.25)
            tol = 24 * U
            near(o[torch.from_numpy(live)], want_o, tol + (2.0 ** -8 if dtype == BF16 else 0), "o")
            assert (o[torch.from_numpy(~live)] == 0).all()
            near(state[at[live].cuda()], want, tol, "state")
            rest = torch.ones(rows + 5, dtype=torch.bool)
            rest[at[live]] = False
            assert torch.equal(state.cpu()[rest], pool[rest])


def test_step_of_states_that_are_not_16_byte_aligned():
    require_gpu()
    x = make(1, 3, 2, 1, 32, 32, F32, 12)
    q, k, v, g, beta = (x[n][0].contiguous().cuda() for n in ("q", "k", "v", "g", "beta"))
    flat = torch.randn(3 * 2 * 32 * 32 + 1, device="cuda")
    one, two = flat[:-1].clone().view(3, 2, 32, 32), torch.empty_like(flat)[1:].view(3, 2, 32, 32)
    two.copy_(one)
    outs = []
    for state in (one, two):
        outs.append(torch.empty_like(v))
        dd.distdl_delta_step(q, k, v, g, beta, state, None, outs[-1], 1.0)
    near(outs[1], outs[0].double().cpu().numpy(), 24 * U, "o")
    near(two, one.double().cpu().numpy(), 24 * U, "state")


def test_steps_are_what_the_chunks_compute():
    require_gpu()
    x = make(2, 70, 4, 2, 64, 48, F32, 13)
    want = run(x, None, 2, 0.3, back=False)
    state, o = x["h0"].cuda().clone(), torch.empty_like(x["v"]).cuda()
    for t in range(70):
        q, k, v, g, beta = (x[n][:, t].contiguous().cuda() for n in ("q", "k", "v", "g", "beta"))
        one = torch.empty_like(v)
        dd.distdl_delta_step(q, k, v, g, beta, state, None, one, 0.3)
        o[:, t] = one
    near(o, want["o"].double().cpu().numpy(), limit(o, 70) + 70 * 2 * U, "o")
    near(state, want["hT"].double().cpu().numpy(), limit(state, 70) + 70 * 2 * U, "hT")


def test_unaligned_tensors():
    """Every tensor starts one element into its allocation."""
    require_gpu()
    for dtype in (F32, BF16):
        x = make(2, 70, 2, 1, 31, 24, dtype, 14)
        want = run(x, None, 1, 0.3)
        def moved(t):
            flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
            flat[1:].copy_(t.reshape(-1))
            return flat[1:].view(t.shape)
        y = {n: moved(t) for n, t in x.items()}
        plan = dd.distdl_delta_plan_create(2, 70, 2, 1, 31, 24, 1, 0.3, dtype)
        o, hT = moved(torch.zeros_like(x["v"])), moved(torch.zeros_like(x["h0"]))
        ins = [[y[n]] for n in ("q", "k", "v", "g", "beta")]
        dd.distdl_delta_fwd(plan, *ins, y["h0"], None, [o], hT)
        assert torch.equal(o, want["o"]) and torch.equal(hT, want["hT"])
        d = {n: moved(torch.zeros_like(x[n])) for n in ("q", "k", "v", "g", "beta")}
        dh0 = moved(torch.zeros_like(x["h0"]))
        dd.distdl_delta_bwd(plan, *ins, y["h0"], None, [y["do"]], y["dhT"], *[[d[n]] for n in ("q", "k", "v", "g", "beta")], dh0)
        for n in d:
            assert torch.equal(d[n], want["d" + n]), n
        assert torch.equal(dh0, want["dh0"])


def test_streams_and_graphs():
    """Calls on two streams at once, and a recorded forward and backward pass replayed on new contents, eager work between the replays."""
    require_gpu()
    shape = (2, 140, 4, 2, 64, 64)
    plan = dd.distdl_delta_plan_create(*shape, 2, 0.3, BF16)
    ins = []
    for seed in (1, 2):
        x = make(*shape, BF16, seed)
        ins.append({n: cut(x[n], 2) for n in ("q", "k", "v", "g", "beta", "do")} | {n: [x[n].cuda()] for n in ("h0", "dhT")})

    def new(x):
        return {n: [torch.zeros_like(t) for t in x[n]] for n in ("q", "k", "v", "g", "beta", "do", "h0", "dhT")}

    def call(x, out):
        dd.distdl_delta_fwd(plan, x["q"], x["k"], x["v"], x["g"], x["beta"], x["h0"][0], None, out["do"], out["dhT"][0])
        dd.distdl_delta_bwd(plan, x["q"], x["k"], x["v"], x["g"], x["beta"], x["h0"][0], None, x["do"], x["dhT"][0], out["q"], out["k"], out["v"],
                            out["g"], out["beta"], out["h0"][0])

    flat = lambda out: [t for ts in out.values() for t in ts]  # noqa: E731
    want = [new(x) for x in ins]
    for x, out in zip(ins, want):
        call(x, out)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [new(x) for x in ins]
    for _ in range(3):
        for st, x, out in zip(streams, ins, got):
            with torch.cuda.stream(st):
                call(x, out)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(u, v) for u, v in zip(flat(a), flat(b)))
    buf, out = {n: [t.clone() for t in ts] for n, ts in ins[0].items()}, new(ins[0])
    with torch.cuda.stream(streams[0]):
        call(buf, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        call(buf, out)
    for i in (1, 0, 1):
        for t, u in zip(flat(buf), flat(ins[i])):
            t.copy_(u)
        for t in flat(out):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(flat(want[i]), flat(out)))


def test_a_first_call_is_refused_while_its_stream_is_captured():
    require_gpu()
    x = make(1, 40, 1, 1, 16, 16, F32)
    c = {n: cut(x[n], 1) for n in ("q", "k", "v", "g", "beta")}
    plan, o, graph = dd.distdl_delta_plan_create(1, 40, 1, 1, 16, 16, 1, 1.0, F32), [torch.zeros_like(c["v"][0])], torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        o[0].add_(1.0)
        with pytest.raises(dd.DistdlError) as e:
            dd.distdl_delta_fwd(plan, c["q"], c["k"], c["v"], c["g"], c["beta"], None, None, o, None)
        assert e.value.code == dd.ERR_INVALID_ARG
    graph.replay()
    torch.cuda.synchronize()
    assert (o[0] == 1.0).all()
