"""Operators of rows of logits on the GPU against the oracle in fp64.

Tolerances.  u = 2^-24.  A log probability is ln 2 (fma(x, c, -mc) - log2 s): the fma and log2 round once each, relative to numbers up to
|z| c, s is a sum of exps that are off by 2 u and by u |d| each, and lanes' partial sums of up to 64 terms in a row; with |z| <= 50 (75 in
units of log 2) each of five such roundings is below 75 u = 4.5e-6.  So 2e-5 absolute covers lse, logp and top; the entropy's w / s is of
terms d e whose relative error is about 10 u, with d up to 20 where e counts: 2e-5 as well.  Gradients: p is off by 75 u + 4 u = 5e-6
relative, each, so 2e-5 of the row's largest magnitude for fp32; bf16 rounds by 2^-8 / 2 of the number itself, on top."""
import numpy as np
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from oracle import tokens

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TOL = 2e-5


def cut(x, parts):
    n = x.shape[1]
    return [t.contiguous() for t in x.split([n // parts + (r < n % parts) for r in range(parts)], 1)]


def make(rows, n_v, dtype, seed=0, masked=0.02, size=3.0):
    g = torch.Generator().manual_seed(seed)
    x = size * torch.randn(rows, n_v, generator=g)
    x[torch.rand(rows, n_v, generator=g) < masked] = -torch.inf
    x = x.to(dtype)
    targets = torch.randint(0, n_v, (rows,), generator=g, dtype=torch.int32)
    if rows > 2:
        targets[1] = -1
    return x, targets, g


def near(got, want, size, what):
    """|got - want| <= size wherever want is finite, the same infinities elsewhere."""
    got, want = got.double().cpu().numpy(), np.asarray(want)
    ends = np.isfinite(want)
    assert np.array_equal(got[~ends], want[~ends]), what
    off = np.abs(got[ends] - want[ends]) - np.broadcast_to(size, want.shape)[ends]
    assert off.size == 0 or off.max() <= 0, f"{what}: {off.max():.3e} over"


def forward(x, targets, parts, k, temperature=1.0, dtype=None):
    rows = x.shape[0]
    plan = dd.distdl_logits_plan_create(rows, x.shape[1], parts, x.dtype)
    new = lambda *s, kind=F32: torch.full(s, -7, dtype=kind, device="cuda")  # noqa: E731
    out = new(rows), new(rows), new(rows), new(rows, k, kind=torch.int32) if k else None, new(rows, k) if k else None
    dd.distdl_logprob_fwd(plan, cut(x.cuda(), parts), targets.cuda(), *out, temperature)
    return plan, out


def check_forward(x, targets, parts, k, temperature=1.0):
    _, (logp, lse, entropy, ids, top) = forward(x, targets, parts, k, temperature)
    want = tokens.logprob_forward(x.double().numpy(), targets.numpy(), k, temperature)
    near(logp, want[0], TOL, "logp")
    near(lse, want[1], TOL, "lse")
    near(entropy, want[2], TOL, "entropy")
    if k:
        assert np.array_equal(ids.cpu().numpy(), want[3])
        near(top, want[4], TOL, "top")


SIZES = [(1, 1, 1, 1), (1, 7, 1, 7), (3, 9, 2, 5), (5, 64, 3, 64), (4, 511, 1, 20), (3, 2048, 4, 64), (2, 8193, 3, 33), (7, 20011, 8, 5),
         (2, 131072, 1, 20), (600, 333, 3, 4), (513, 4099, 2, 64), (3, 100, 33, 12), (600, 40, 20, 3)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, n_v, parts, k", SIZES)
def test_forward(rows, n_v, parts, k, dtype):
    require_gpu()
    x, targets, _ = make(rows, n_v, dtype)
    check_forward(x, targets, parts, k)


@pytest.mark.parametrize("temperature", [0.5, 3.0])
def test_forward_with_a_temperature_and_without_alternatives(temperature):
    require_gpu()
    for dtype in (F32, BF16):
        x, targets, _ = make(9, 5003, dtype, 3)
        check_forward(x, targets, 2, 0, temperature)
        check_forward(x, targets, 2, 9, temperature)


@pytest.mark.parametrize("rows", [2, 520])
def test_equal_values_keep_their_order(rows):
    """Constant rows, two values, and rows that rise and fall: every wave's threshold is met again and again."""
    require_gpu()
    n = 9001
    g = torch.Generator().manual_seed(1)
    ramp = torch.linspace(-20, 20, n)
    kinds = [torch.zeros(n), torch.randint(0, 2, (n,), generator=g).float(), ramp, ramp.flip(0), -torch.zeros(n), torch.where(torch.arange(n) % 3 == 0, -0.0, 0.0)]
    x = torch.stack([kinds[r % len(kinds)] for r in range(rows)])
    for dtype in (F32, BF16):
        y = x.to(dtype)
        for k in (1, 40, 64):
            _, (_, _, _, ids, _) = forward(y, torch.zeros(rows, dtype=torch.int32), 3, k)
            want = np.argsort(-(y.double().numpy() + 0.0), axis=1, kind="stable")[:, :k]
            assert np.array_equal(ids.cpu().numpy(), want)


def test_rows_that_masks_leave_nothing_or_little():
    require_gpu()
    for dtype in (F32, BF16):
        x = torch.full((6, 3001), -torch.inf, dtype=dtype)
        x[1, 2999] = 3.0
        x[2, [5, 6, 2000]] = torch.tensor([1.0, 1.0, 2.0], dtype=dtype)
        x[3] = torch.finfo(dtype).min  # a mask of the lowest value: all entries alike
        x[4, ::2] = torch.finfo(dtype).min
        x[4, 100] = 0.0
        targets = torch.tensor([4, 2999, 0, 7, 100, 3001], dtype=torch.int32)
        plan, (logp, lse, entropy, ids, top) = forward(x, targets, 2, 6)
        want = tokens.logprob_forward(x[:3].double().numpy(), targets[:3].numpy(), 6)
        near(logp[:3], want[0], TOL, "logp")
        near(lse[:3], want[1], TOL, "lse")
        near(entropy[:3], want[2], TOL, "entropy")
        assert np.array_equal(ids[:3].cpu().numpy(), want[3])
        near(top[:3], want[4], TOL, "top")
        near(entropy[3:5], [np.log(3001.0), 0.0], TOL, "entropy")
        near(logp[4:5], [0.0], TOL, "logp")
        assert logp[5] == 0.0
        # gradients: zeros for the empty row, whatever its gradient
        dx = [torch.full_like(t, 7.0) for t in cut(x.cuda(), 2)]
        ones = torch.ones(6, device="cuda")
        dd.distdl_logprob_bwd(plan, cut(x.cuda(), 2), targets.cuda(), lse, entropy, ones, ones, dx)
        got = torch.cat(dx, 1).double().cpu().numpy()
        assert (got[0] == 0).all()
        want = tokens.logprob_adjoint(x[1:3].double().numpy(), targets[1:3].numpy(), np.ones(2), np.ones(2))
        assert np.abs(got[1:3] - want).max() <= TOL + 2.0 ** -8


def test_infinities_and_nans_answer_nan_and_leave_other_rows_alone():
    require_gpu()
    x, targets, _ = make(4, 5000, F32, 5, masked=0)
    clean = tokens.logprob_forward(x.double().numpy(), targets.numpy(), 8)
    x[1, 4321] = torch.nan
    x[2, 17] = torch.inf
    _, (logp, lse, entropy, ids, top) = forward(x, targets, 3, 8)
    for r in (1, 2):
        assert torch.isnan(lse[r]) and torch.isnan(entropy[r])
    for r in (0, 3):
        near(lse[r], clean[1][r], TOL, "lse")
        assert np.array_equal(ids[r].cpu().numpy(), clean[3][r])
    want = np.argsort(-np.nan_to_num(x[1].double().numpy(), nan=-np.inf), kind="stable")[:8]
    assert np.array_equal(ids[1].cpu().numpy(), want)  # a NaN is no alternative
    few = torch.full((1, 5), torch.nan)
    few[0, 3] = 1.0
    _, (_, _, _, ids, _) = forward(few, torch.zeros(1, dtype=torch.int32), 1, 3)
    assert ids[0].tolist() == [3, -1, -1]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, n_v, parts", [(1, 1, 1), (3, 5, 2), (5, 1001, 3), (2, 70001, 2), (530, 700, 3), (3, 100, 33)])
@pytest.mark.parametrize("what", ["logp", "entropy", "both"])
def test_adjoint(rows, n_v, parts, dtype, what):
    require_gpu()
    x, targets, g = make(rows, n_v, dtype, 2)
    dlogp, dent = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    if rows > 4:
        dlogp[2] = 0.0
    want = tokens.logprob_adjoint(x.double().numpy(), targets.numpy(), dlogp.double().numpy() * (what != "entropy"),
                                  dent.double().numpy() * (what != "logp"), 0.8)
    plan, (_, lse, entropy, _, _) = forward(x, targets, parts, 0, 0.8)
    x_ = cut(x.cuda(), parts)
    dx = [torch.full_like(t, 7.0) for t in x_]
    args = (targets.cuda(), lse, entropy if what != "logp" else None, dlogp.cuda() if what != "entropy" else None, dent.cuda() if what != "logp" else None)
    dd.distdl_logprob_bwd(plan, x_, *args, dx, 0.8)
    got = torch.cat(dx, 1)
    size = np.abs(want).max(1, keepdims=True)
    # (log p + H is off by 4e-5 at most, p's own gradient of the entropy is up to |log p| times as large as what is left of it)
    near(got, want, 12 * TOL * size + 1e-7 + (2.0 ** -8 * np.abs(want) if dtype == BF16 else 0), "dx")
    dd.distdl_logprob_bwd(plan, x_, *args, x_, 0.8)  # in place
    assert torch.equal(torch.cat(x_, 1), got)


def test_adjoint_is_the_derivative():
    """Central differences of the oracle's forward pass, whose adjoint the kernels are held against."""
    rng = np.random.default_rng(0)
    x, t, w, e = rng.normal(size=(3, 12)), np.array([2, -1, 11]), rng.normal(size=3), rng.normal(size=3)

    def value(x):
        logp, _, entropy, _, _ = tokens.logprob_forward(x, t, 0, 0.7)
        return (np.where(t >= 0, w, 0) * logp + e * entropy).sum()
    got = tokens.logprob_adjoint(x, t, w, e, 0.7)
    for i in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[i] = 1e-5
        assert abs((value(x + d) - value(x - d)) / 2e-5 - got[i]) < 1e-8


def teacher_of(rows, n_v, k, g):
    ids = torch.stack([torch.randperm(n_v, generator=g)[:k] if k <= n_v else torch.randint(0, n_v, (k,), generator=g) for _ in range(rows)]).to(torch.int32)
    return ids, 2 * torch.randn(rows, k, generator=g)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows, n_v, parts, k", [(1, 1, 1, 1), (3, 5, 2, 5), (4, 1001, 3, 17), (2, 70001, 2, 64), (530, 700, 3, 300), (3, 100, 33, 9), (2, 3000, 2, 1024)])
def test_distill(rows, n_v, parts, k, dtype):
    """The loss is a sum of t (log t - log p): 2e-5 for each logarithm, the t sum to 1.  A row whose entries the student cannot answer with is infinite."""
    require_gpu()
    x, _, g = make(rows, n_v, dtype, 4, masked=0.002)
    ids, teacher = teacher_of(rows, n_v, k, g)
    weight = torch.rand(rows, generator=g)
    if rows > 2:
        ids[0, k // 2:] = -1
        ids[1] = ids[1, :1].clone() if k < 2 else ids[1, torch.arange(k) // 2]  # every place twice
        ids[2, 0], weight[2] = n_v, 0.0
    want_loss, want = tokens.distill(x.double().numpy(), ids.numpy(), teacher.double().numpy(), weight.double().numpy(), 1.5)
    plan, x_ = dd.distdl_logits_plan_create(rows, n_v, parts, dtype), cut(x.cuda(), parts)
    loss, dx = torch.full((rows,), 7.0, device="cuda"), [torch.full_like(t, 7.0) for t in x_]
    args = (ids.cuda(), teacher.cuda(), weight.cuda())
    dd.distdl_distill_fwd_bwd(plan, x_, *args, loss, dx, 1.5)
    near(loss, want_loss, 2 * TOL, "loss")
    got = torch.cat(dx, 1)
    size = np.abs(want).max(1, keepdims=True)
    near(got, want, TOL * size + 1e-7 + (2.0 ** -8 * np.abs(want) if dtype == BF16 else 0), "dx")
    alone = torch.full((rows,), 7.0, device="cuda")
    dd.distdl_distill_fwd_bwd(plan, x_, *args, alone, None, 1.5)
    assert torch.equal(alone, loss)
    dd.distdl_distill_fwd_bwd(plan, x_, *args, None, x_, 1.5)  # in place
    assert torch.equal(torch.cat(x_, 1), got)


def test_distill_rows_without_a_teacher_or_a_student():
    require_gpu()
    x, _, g = make(5, 2000, F32, 6, masked=0)
    ids, teacher = teacher_of(5, 2000, 8, g)
    ids[0] = -1
    teacher[1] = -torch.inf
    x[2] = -torch.inf
    x[0, 7] = torch.nan  # of a row that nothing is taken from
    x[3, 9] = torch.nan
    plan, x_ = dd.distdl_logits_plan_create(5, 2000, 2, F32), cut(x.cuda(), 2)
    loss, dx = torch.full((5,), 7.0, device="cuda"), [torch.full_like(t, 7.0) for t in x_]
    dd.distdl_distill_fwd_bwd(plan, x_, ids.cuda(), teacher.cuda(), None, loss, dx)
    dx = torch.cat(dx, 1)
    assert loss[0] == 0 and loss[1] == 0 and torch.isinf(loss[2]) and torch.isnan(loss[3])
    assert (dx[:3] == 0).all() and torch.isfinite(dx[4]).all()
    want_loss, want = tokens.distill(x[4:].double().numpy(), ids[4:].numpy(), teacher[4:].double().numpy(), np.ones(1))
    near(loss[4:], want_loss, 2 * TOL, "loss")
    near(dx[4:], want, TOL, "dx")


def test_one_place_is_the_cross_entropy():
    require_gpu()
    x, targets, _ = make(6, 3000, F32, 7, masked=0)
    targets[1] = 5
    plan, x_ = dd.distdl_logits_plan_create(6, 3000, 1, F32), [x.cuda()]
    loss, dx = torch.empty(6, device="cuda"), [torch.empty_like(x_[0])]
    dd.distdl_distill_fwd_bwd(plan, x_, targets.cuda()[:, None].contiguous(), torch.full((6, 1), -3.0, device="cuda"), None, loss, dx)
    _, (logp, lse, _, _, _) = forward(x, targets, 1, 0)
    other = [torch.empty_like(x_[0])]
    dd.distdl_logprob_bwd(plan, x_, targets.cuda(), lse, None, torch.full((6,), -1.0, device="cuda"), None, other)
    near(loss, -logp.double().cpu().numpy(), TOL, "loss")
    near(dx[0], other[0].double().cpu().numpy(), TOL, "dx")


@pytest.mark.parametrize("rows", [3, 600])
def test_streams_and_graphs(rows):
    """Calls on two streams at once; recorded and replayed on new contents, eager work between the replays."""
    require_gpu()
    n_v, k = 30011, 7
    xs = [make(rows, n_v, BF16, s)[0] for s in (1, 2)]
    targets = make(rows, n_v, BF16, 1)[1].cuda()
    ids, teacher = (t.cuda() for t in teacher_of(rows, n_v, k, torch.Generator().manual_seed(3)))
    plan = dd.distdl_logits_plan_create(rows, n_v, 2, BF16)

    def call(x, out):
        dd.distdl_logprob_fwd(plan, x, targets, *out[:5])
        dd.distdl_logprob_bwd(plan, x, targets, out[1], out[2], out[0], out[2], out[5])
        dd.distdl_distill_fwd_bwd(plan, x, ids, teacher, None, out[6], out[7])

    def new(x):
        return [torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"),
                torch.empty(rows, k, dtype=torch.int32, device="cuda"), torch.empty(rows, k, device="cuda"), [torch.empty_like(t) for t in x],
                torch.empty(rows, device="cuda"), [torch.empty_like(t) for t in x]]

    # (bits: a target of -inf has a gradient of -inf here, and its row NaNs)
    flat = lambda out: [t.view(torch.int16 if t.dtype == BF16 else torch.int32) for o in out for t in (o if isinstance(o, list) else [o])]  # noqa: E731
    ins = [cut(x.cuda(), 2) for x in xs]
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
    buf, out = [t.clone() for t in ins[0]], new(ins[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(streams[0]):
        call(buf, out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=streams[0]):
        call(buf, out)
    for i in (1, 0, 1):
        for t, u in zip(buf, ins[i]):
            t.copy_(u)
        for t in flat(out):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(flat(want[i]), flat(out)))


def test_a_first_call_that_needs_scratch_is_refused_while_its_stream_is_captured():
    require_gpu()
    x, targets, _ = make(2, 30000, F32)
    plan, x, targets = dd.distdl_logits_plan_create(2, 30000, 1, F32), [x.cuda()], targets.cuda()
    lse, graph = torch.zeros(2, device="cuda"), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lse.add_(1.0)
        with pytest.raises(dd.DistdlError) as e:
            dd.distdl_logprob_fwd(plan, x, targets, None, lse, None)
        assert e.value.code == dd.ERR_INVALID_ARG
    graph.replay()
    torch.cuda.synchronize()
    assert (lse == 1.0).all()


def test_no_rows():
    require_gpu()
    plan = dd.distdl_logits_plan_create(0, 100, 2, F32)
    x, none = [torch.empty(0, 50, device="cuda")] * 2, torch.empty(0, device="cuda")
    dd.distdl_logprob_fwd(plan, x, none.int(), none, none, none)
    dd.distdl_logprob_bwd(plan, x, none.int(), none, none, none, none, x)
    dd.distdl_distill_fwd_bwd(plan, x, torch.empty(0, 3, dtype=torch.int32, device="cuda"), torch.empty(0, 3, device="cuda"), None, none, x)
