"""The norm's answers follow from its own row factors: n = s rstd, rounded, is what the gain multiplies, in the answer as in the adjoint."""
import numpy as np
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from oracle import blocks
from test_gpu_norm import KINDS, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n_f,P", [(3, 8, 1), (7, 513, 2), (4, 1001, 3), (40, 4096, 2), (9, 9000, 1), (2, 20000, 1)])
def test_answers_from_the_row_factors(rows, n_f, P, dtype):
    """To the bit, in the type and in 8-bit blocks, from the unrounded sum."""
    require_gpu()
    (x, r, _, _), g = make(rows, n_f, P, dtype, seed=6)
    plan = dd.distdl_rmsnorm_plan_create(rows, n_f, P, 1e-5, KINDS[dtype])
    y, rstd = [torch.empty_like(t) for t in x], torch.empty(rows, device="cuda")
    q = [torch.empty(t.shape, dtype=torch.uint8, device="cuda") for t in x]
    qs = [torch.empty(-(-t.shape[1] // 128), rows, dtype=torch.uint8, device="cuda") for t in x]
    dd.distdl_rmsnorm_fwd(plan, x, r, g, None, y, q, qs, rstd)
    for j in range(P):
        want = (x[j].float() + r[j].float()) * rstd[:, None] * g[j]
        assert torch.equal(y[j], want.to(KINDS[dtype]))
        codes, scales = blocks.quantise(want.double().cpu().numpy(), 1, 128)
        assert np.array_equal(qs[j].cpu().numpy().T, scales) and np.array_equal(q[j].cpu().numpy(), codes)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [1e-30, 1e-42, 1e-60])
def test_rows_of_zeros_under_a_tiny_eps(eps, dtype):
    """Rows of zeros (masked ones) answer zeros, and their gradients are finite, for an eps that 32 bits do not hold either."""
    require_gpu()
    rows, n_f, P = 6, 700, 2
    (x, dy, _, _), g = make(rows, n_f, P, dtype, seed=7)
    for t in x:
        t[::2] = 0
    for t in dy:
        t[::2] = 0
    plan = dd.distdl_rmsnorm_plan_create(rows, n_f, P, eps, KINDS[dtype])
    y, rstd = [torch.empty_like(t) for t in x], torch.empty(rows, device="cuda")
    dd.distdl_rmsnorm_fwd(plan, x, None, g, None, y, None, None, rstd)
    assert torch.isfinite(rstd).all()
    dx, dg = [torch.empty_like(t) for t in x], [torch.empty_like(t) for t in g]
    dd.distdl_rmsnorm_bwd(plan, x, g, rstd, dy, None, dx, dg)
    for t in y + dx:
        assert not t[::2].any() and torch.isfinite(t).all() and t[1::2].any()
    assert all(torch.isfinite(t).all() for t in dg)
