"""8-bit products whose operands share memory, and every kind of tile with the operands that are hard for it."""
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from test_gpu_linear8 import KINDS, ceil8, empty8, quantised

pytestmark = pytest.mark.gpu


def coded(seed, rows, cols, tiles=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, s = empty8(rows, cols, tiles)
    dd.distdl_quant8([torch.randn(rows, cols, generator=g, device="cuda")], [q], [s], None, None, tiles=tiles)
    return q, s


@pytest.mark.parametrize("n_b", [131, 128, 1000, 2051])
@pytest.mark.parametrize("fo,fi", [(80, 300), (300, 80), (200, 201)])
def test_weight_gradient_of_operands_at_one_address(fo, fi, n_b):
    """dW of a matrix's first rows with the whole matrix: both operands start at one address and have different numbers of rows."""
    require_gpu()
    most = max(fo, fi)
    q, s = coded(1, most, n_b)
    scales = lambda rows: s[:, :rows].contiguous()  # noqa: E731
    plan = dd.distdl_linear8_plan_create(n_b, fi, fo, 1, 1, torch.float32)
    dw = [torch.full((fo, fi), 7.0, device="cuda") for _ in range(2)]
    dd.distdl_linear8_bwd_w(plan, [q[:fo]], [scales(fo)], [q[:fi]], [scales(fi)], [dw[0]])
    dd.distdl_linear8_bwd_w(plan, [q[:fo].clone()], [scales(fo)], [q[:fi].clone()], [scales(fi)], [dw[1]])
    assert torch.equal(*dw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n_b", [40, 100, 700])
def test_workers_of_different_widths_at_one_address(n_b, dtype):
    """Two workers of 167 and 166 features whose inputs, and whose weights, are views of one buffer each: rows of different length from one address."""
    require_gpu()
    n_fi, n_fo, fi, fo = 333, 401, [167, 166], [201, 200]
    x, w = coded(2, n_b, 167), coded(3, 201, 167, tiles=True)
    view = lambda t, r, c: t.view(-1)[:r * c].view(r, c)  # noqa: E731
    xs = [x[1][:, :n_b]] * 2
    plan = dd.distdl_linear8_plan_create(n_b, n_fi, n_fo, 2, 2, KINDS[dtype])
    y = [[torch.empty(n_b, m, dtype=KINDS[dtype], device="cuda") for m in fo] for _ in range(2)]
    for clone, out in zip((False, True), y):
        own = (lambda t: t.clone()) if clone else (lambda t: t)  # noqa: E731
        dd.distdl_linear8_fwd(plan, [own(view(x[0], n_b, c)) for c in fi], xs, [own(view(w[0], m, c)) for m in fo for c in fi], [w[1]] * 4, out)
    assert all(torch.equal(a, b) for a, b in zip(*y))
    assert ceil8(167) == ceil8(166) and ceil8(201) == ceil8(200)


def held(y, pairs, dtype):
    """Against the sum in 64 bits.  fp32 results: each of the K / 32 steps of a sum cuts off one unit of 2^-23 at most of the sum of
    magnitudes.  bf16 results: 2^-8 of themselves, and 2^-10 of the sum of each eight neighbouring products' largest, which the codes' own instruction may cut off."""
    pairs = [(torch.tensor(a, device="cuda"), torch.tensor(b, device="cuda")) for a, b in pairs]
    want = sum(a @ b.t().contiguous() for a, b in pairs)
    if dtype == "f32":
        tol = (sum(a.shape[1] for a, _ in pairs) / 32 + 4 * len(pairs)) * 2.0 ** -23 * sum(a.abs() @ b.abs().t().contiguous() for a, b in pairs)
    else:
        tol = 2.0 ** -8 * want.abs()
        for a, b in pairs:
            for k in range(0, a.shape[1], 8):
                most = torch.zeros_like(want)
                for i in range(k, min(k + 8, a.shape[1])):
                    torch.maximum(most, a[:, i, None].abs() * b[None, :, i].abs(), out=most)
                tol += 2.0 ** -10 * most
    bad = torch.isnan(want)
    assert torch.equal(torch.isnan(y), bad)
    off = ~((y.double() - want).abs() <= tol) & ~bad
    assert not off.any(), f"{int(off.sum())} of {off.numel()} off"


# Rows and columns whose cheapest tiles are, by what a round of 256 of them takes, 64 x 64 (bf16 and fp32), 128 x 128 (both), and 256 x 256 (bf16) or 256 x 128 (fp32).
@pytest.mark.parametrize("moved", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(300, 520), (1000, 2040), (4096, 4090)], ids=["64", "128", "256"])
def test_every_tile_with_hard_operands(m, n, dtype, moved):
    """Two workers of the sum with 167 and 166 features (moved: 160 each, one byte into an allocation), a NaN in one row, an infinity in one tile; and
    the weight gradient of the same operands, whose sum has those lengths."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(m)
    rnd = lambda r, c: torch.randn(r, c, generator=g, device="cuda") * torch.exp(torch.randn(r, 1, generator=g, device="cuda"))  # noqa: E731
    shift = (lambda t: torch.cat([torch.zeros(1, dtype=t.dtype, device="cuda"), t.reshape(-1)])[1:].view(t.shape)) if moved else (lambda t: t)
    widths = [160, 160] if moved else [167, 166]
    x, w = [rnd(m, c) for c in widths], [rnd(n, c) for c in widths]
    x[0][1, 3], w[1][200, 130] = float("nan"), float("inf")
    xq, wq = [quantised(t) for t in x], [quantised(t, tiles=True) for t in w]
    plan = dd.distdl_linear8_plan_create(m, sum(widths), n, 1, 2, KINDS[dtype])
    y = torch.full((m, n), 7.0, dtype=KINDS[dtype], device="cuda")
    dd.distdl_linear8_fwd(plan, [shift(t[0]) for t in xq], [t[1] for t in xq], [shift(t[0]) for t in wq], [t[1] for t in wq], [y])
    held(y, [(a[2], b[2]) for a, b in zip(xq, wq)], dtype)
    if dtype == "f32":
        k = widths[0]
        a, b = rnd(m, k), rnd(n, k)
        a[1, 3], b[200, 130] = float("nan"), float("inf")
        aq, bq = quantised(a), quantised(b)
        plan = dd.distdl_linear8_plan_create(k, n, m, 1, 1, torch.float32)
        dw = torch.full((m, n), 7.0, device="cuda")
        dd.distdl_linear8_bwd_w(plan, [shift(aq[0])], [aq[1]], [shift(bq[0])], [bq[1]], [dw])
        held(dw, [(aq[2], bq[2])], "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(4, 64), (40, 64), (300, 520), (1000, 2040), (4096, 4090)])
def test_operands_below_the_normal_numbers(m, n, dtype):
    """Numbers down to 2^-133 count in full where the other operand brings their products back into range."""
    require_gpu()
    x, w = torch.zeros(m, 128, device="cuda"), torch.zeros(n, 128, device="cuda")
    size = (torch.arange(m, device="cuda") % 15 + 1).double()
    x[:, 0] = (size * 2.0 ** -133).float()
    w[:, 0] = 2.0 ** 100
    xq, wq = quantised(x), quantised(w, tiles=True)
    plan = dd.distdl_linear8_plan_create(m, 128, n, 1, 1, KINDS[dtype])
    y = torch.empty(m, n, dtype=KINDS[dtype], device="cuda")
    dd.distdl_linear8_fwd(plan, [xq[0]], [xq[1]], [wq[0]], [wq[1]], [y])
    assert torch.equal(y.double(), (size * 2.0 ** -33)[:, None].expand(m, n))
