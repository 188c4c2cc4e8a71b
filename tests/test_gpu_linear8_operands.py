"""8-bit products whose operands share memory, and every kind of tile with the operands that are hard for it."""
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from test_gpu_linear8 import KINDS, ceil8, empty8

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
