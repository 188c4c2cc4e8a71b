"""Root-mean-square norm with the residual's addition on the GPU against the fp64 oracle.

Tolerances.  A row's sum of squares is at most 32 fused steps a thread and 10 of the tree, all terms positive, so rstd is off by at most
(42 / 2 + 2) units of 2^-24; y has three roundings more.  32 units (2^-19) hold for y, and for dx against the sizes of its
terms.  dg sums `rows` products: its error is held against the sum of their magnitudes, (rows + 64) units."""
import numpy as np
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from oracle import blocks

pytestmark = pytest.mark.gpu
UNIT = 2.0 ** -24
HALF_BF16 = 2.0 ** -8
KINDS = {"f32": torch.float32, "bf16": torch.bfloat16}


def cut(x, P):
    sizes = [x.shape[-1] // P + (r < x.shape[-1] % P) for r in range(P)]
    return [t.contiguous() for t in x.split(sizes, -1)]


def wide(ts):
    return torch.cat([t.float() for t in ts], -1).cpu().double().numpy()


def within(got, want, tol):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, the first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}"


def make(rows, n_f, P, dtype, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = KINDS[dtype]
    x = [(scale * torch.randn(rows, n_f, generator=g, device="cuda")).to(t) for _ in range(4)]
    gain = 1 + 0.2 * torch.randn(n_f, generator=g, device="cuda")
    return [cut(v, P) for v in x], cut(gain, P)


SIZES = [(1, 1, 1), (3, 8, 1), (5, 130, 3), (2, 512, 1), (7, 513, 2), (4, 1001, 3), (9, 2048, 1), (3, 2055, 4), (6, 4096, 2), (2, 8191, 3),
         (3, 9000, 2), (2, 20000, 1), (5, 300, 11), (1100, 96, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n_f,P", SIZES)
def test_forward(rows, n_f, P, dtype):
    require_gpu()
    (x, r, _, _), g = make(rows, n_f, P, dtype)
    plan = dd.distdl_rmsnorm_plan_create(rows, n_f, P, 1e-5, KINDS[dtype])
    for res in (None, r):
        s, y = [torch.empty_like(t) for t in x], [torch.empty_like(t) for t in x]
        rstd = torch.empty(rows, device="cuda")
        dd.distdl_rmsnorm_fwd(plan, x, res, g, s, y, None, None, rstd)
        ws, wy, wr = blocks.norm_forward(wide(x), None if res is None else wide(res), wide(g), 1e-5)
        half = HALF_BF16 if dtype == "bf16" else UNIT
        within(wide(s), ws, half * np.abs(ws))
        within(wide(y), wy, (half + 32 * UNIT) * np.abs(wy))
        within(rstd.cpu().double().numpy(), wr, 32 * UNIT * wr)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n_f,P", SIZES)
def test_answer_in_8_bits(rows, n_f, P, dtype):
    """Codes and scales are those of the oracle's y but for ties and block maxima that y's own error moves."""
    require_gpu()
    (x, r, _, _), g = make(rows, n_f, P, dtype, seed=1)
    plan = dd.distdl_rmsnorm_plan_create(rows, n_f, P, 1e-5, KINDS[dtype])
    q = [torch.empty(t.shape, dtype=torch.float8_e4m3fn, device="cuda") for t in x]
    qs = [torch.empty(-(-t.shape[1] // 128), rows, dtype=torch.uint8, device="cuda") for t in x]
    dd.distdl_rmsnorm_fwd(plan, x, r, g, None, None, q, qs, None)
    _, wy, _ = blocks.norm_forward(wide(x), wide(r), wide(g), 1e-5)
    at = 0
    for k, t in enumerate(q):
        want = wy[:, at:at + t.shape[1]]
        at += t.shape[1]
        _, bytes_ = blocks.quantise(want, 1, 128)
        got = qs[k].cpu().numpy().T
        assert (np.abs(got.astype(int) - bytes_) <= 1).all() and (got != bytes_).mean() <= 0.01 + 1 / got.size
        value = blocks.values_of(t.view(torch.uint8).cpu().numpy(), got, 1, 128)
        unit = (2.0 ** (got.astype(float) - 127)).repeat(128, 1)[:, :value.shape[1]]
        # half a unit of a three-bit mantissa, or of the smallest code
        within(value, want, np.maximum(np.abs(want) / 16, unit * 2.0 ** -10) + 32 * UNIT * np.abs(want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n_f,P", SIZES)
def test_adjoint(rows, n_f, P, dtype):
    require_gpu()
    (s, dy, ds, _), g = make(rows, n_f, P, dtype, seed=2)
    plan = dd.distdl_rmsnorm_plan_create(rows, n_f, P, 1e-5, KINDS[dtype])
    sw, gw, dyw = wide(s), wide(g), wide(dy)
    _, _, rstd = blocks.norm_forward(sw, None, gw, 1e-5)
    r = torch.tensor(rstd, device="cuda").float()
    r64 = r.cpu().double().numpy()
    for extra in (None, ds):
        dx, dg = [torch.empty_like(t) for t in s], [torch.empty_like(t) for t in g]
        dd.distdl_rmsnorm_bwd(plan, s, g, r, dy, extra, dx, dg)
        wx, wg = blocks.norm_adjoint(sw, gw, r64, dyw, None if extra is None else wide(extra))
        n = sw * r64[:, None]
        terms = r64[:, None] * (np.abs(dyw * gw) + np.abs(n) * np.abs(dyw * gw * n).mean(1, keepdims=True))
        within(wide(dx), wx, (HALF_BF16 if dtype == "bf16" else UNIT) * np.abs(wx) + 64 * UNIT * terms)
        within(wide(dg), wg, (rows + 64) * UNIT * np.abs(dyw * n).sum(0))
        again = [torch.empty_like(t) for t in g]
        dd.distdl_rmsnorm_bwd(plan, s, g, r, dy, extra, dx, again)
        assert all(torch.equal(a, b) for a, b in zip(dg, again)), "a fixed order of sums"


def test_adjoint_is_the_difference_of_the_forward():
    """Along a direction: f32 forward at +- 1/64, differences good to 2^-12 of third derivatives and 2^-17 of rounding."""
    require_gpu()
    rows, n_f, P = 6, 700, 2
    (x, v, dy, _), g = make(rows, n_f, P, "f32", seed=3)
    plan = dd.distdl_rmsnorm_plan_create(rows, n_f, P, 1e-5, torch.float32)
    y = [torch.empty_like(t) for t in x]
    rstd = torch.empty(rows, device="cuda")

    def f(sign):
        dd.distdl_rmsnorm_fwd(plan, [a + sign / 64 * b for a, b in zip(x, v)], None, g, None, y, None, None, rstd)
        return (wide(y) * wide(dy)).sum(1)

    slope = 32 * (f(1) - f(-1))
    f(0)
    dx, dg = [torch.empty_like(t) for t in x], [torch.empty_like(t) for t in g]
    dd.distdl_rmsnorm_bwd(plan, x, g, rstd, dy, None, dx, dg)
    size = np.linalg.norm(wide(dx), axis=1) * np.linalg.norm(wide(v), axis=1)
    within((wide(dx) * wide(v)).sum(1), slope, 1e-3 * size)


def test_special_values_and_offsets():
    require_gpu()
    rows, n_f = 6, 300
    (x, r, _, _), g = make(rows, n_f, 1, "f32", seed=4)
    x[0][1, 5], x[0][2, 7], x[0][3] = float("nan"), float("inf"), 0.0
    x[0][4] = 1e-30
    y, q = torch.empty_like(x[0]), torch.empty(rows, n_f, dtype=torch.uint8, device="cuda")
    qs = torch.empty(3, rows, dtype=torch.uint8, device="cuda")
    plan = dd.distdl_rmsnorm_plan_create(rows, n_f, 1, 1e-5, torch.float32)
    dd.distdl_rmsnorm_fwd(plan, x, None, g, None, [y], [q], [qs], None)
    value = blocks.values_of(q.cpu().numpy(), qs.cpu().numpy().T, 1, 128)
    y = y.cpu().numpy()
    assert np.isnan(y[1]).all() and np.isnan(value[1]).all()          # a NaN in a row is one in its sum
    assert np.isnan(y[2, 7]) and not y[2, :7].any()                    # inf / inf beside finite / inf
    assert not y[3].any() and not value[3].any()                       # a row of zeros stays one
    assert np.isfinite(y[[0, 4, 5]]).all() and np.isfinite(value[[0, 4, 5]]).all()
    # arrays that start at an odd element, bf16
    (a, b, _, _), g = make(3, 257, 1, "bf16", seed=5)
    plan = dd.distdl_rmsnorm_plan_create(3, 257, 1, 1e-5, torch.bfloat16)
    moved = lambda t: torch.cat([torch.zeros(1, dtype=t.dtype, device="cuda"), t.reshape(-1)])[1:].view(t.shape)  # noqa: E731
    y1, y2 = torch.empty_like(a[0]), moved(a[0])
    dd.distdl_rmsnorm_fwd(plan, a, b, g, None, [y1], None, None, None)
    dd.distdl_rmsnorm_fwd(plan, [moved(a[0])], [moved(b[0])], [moved(g[0])], None, [y2], None, None, None)
    assert torch.equal(y1, y2)


def test_in_place_other_stream_and_graph():
    require_gpu()
    rows, n_f, P = 33, 640, 2
    (x, r, dy, _), g = make(rows, n_f, P, "bf16", seed=6)
    plan = dd.distdl_rmsnorm_plan_create(rows, n_f, P, 1e-5, torch.bfloat16)
    new = lambda: [torch.empty_like(t) for t in x]  # noqa: E731
    s, y, rstd = new(), new(), torch.empty(rows, device="cuda")
    dd.distdl_rmsnorm_fwd(plan, x, r, g, s, y, None, None, rstd)
    place = [t.clone() for t in r]
    y2 = new()
    dd.distdl_rmsnorm_fwd(plan, x, place, g, place, y2, None, None, rstd)
    assert all(torch.equal(a, b) for a, b in zip(s + y, place + y2))
    dx, dg = new(), [torch.empty_like(t) for t in g]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        dd.distdl_rmsnorm_bwd(plan, s, g, rstd, dy, None, dx, dg)
    stream.synchronize()
    want = [t.clone() for t in dx + dg]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        dd.distdl_rmsnorm_bwd(plan, s, g, rstd, dy, None, dx, dg)
    for _ in range(3):
        for t in dx + dg:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, dx + dg))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n_f,P", [(7, 513, 2), (9, 2048, 1), (5, 9000, 2), (3, 20000, 1)])
def test_answers_over_their_inputs(rows, n_f, P, dtype):
    """Every lying-over that the calls allow gives the bits of the call with arrays of its own."""
    require_gpu()
    (x, r, dy, ds), g = make(rows, n_f, P, dtype, seed=7)
    plan = dd.distdl_rmsnorm_plan_create(rows, n_f, P, 1e-5, KINDS[dtype])
    new = lambda ts: [torch.empty_like(t) for t in ts]  # noqa: E731
    copy = lambda ts: [t.clone() for t in ts]  # noqa: E731
    same = lambda a, b: all(torch.equal(u, v) for u, v in zip(a, b))  # noqa: E731
    s, y, rstd = new(x), new(x), torch.empty(rows, device="cuda")
    dd.distdl_rmsnorm_fwd(plan, x, r, g, s, y, None, None, rstd)
    for s_on in (0, 1):
        at = [copy(x), copy(r)]
        y2 = new(x)
        dd.distdl_rmsnorm_fwd(plan, at[0], at[1], g, at[s_on], y2, None, None, rstd)
        assert same(s, at[s_on]) and same(y, y2)
        at = [copy(x), copy(r)]
        s2 = new(x)
        dd.distdl_rmsnorm_fwd(plan, at[0], at[1], g, s2, at[s_on], None, None, rstd)
        assert same(s, s2) and same(y, at[s_on])
    dx, dg = new(x), new(g)
    dd.distdl_rmsnorm_bwd(plan, s, g, rstd, dy, ds, dx, dg)
    for dx_on in range(3):
        at = [copy(s), copy(dy), copy(ds)]
        dg2 = new(g)
        dd.distdl_rmsnorm_bwd(plan, at[0], g, rstd, at[1], at[2], at[dx_on], dg2)
        assert same(dx, at[dx_on]) and same(dg, dg2), ("s", "dy", "dsum")[dx_on]


def test_no_rows():
    require_gpu()
    plan = dd.distdl_rmsnorm_plan_create(0, 40, 1, 1e-5, torch.float32)
    e = [torch.empty(0, 40, device="cuda")]
    g, dg, rstd = [torch.ones(40, device="cuda")], [torch.ones(40, device="cuda")], torch.empty(0, device="cuda")
    dd.distdl_rmsnorm_fwd(plan, e, None, g, None, e, None, None, rstd)
    dd.distdl_rmsnorm_bwd(plan, e, g, rstd, e, None, e, dg)
    assert not dg[0].any()
