"""Many rows of logits, which are not cut: rows that are one wave's and rows that are a workgroup's, of every kernel, against the oracle in fp64.

Tolerances as in test_gpu_logits.py: a lane adds up to 512 numbers one behind the other in every one of these calls, positive ones, each sum off by half a step of what
is summed so far: 256 u = 1.5e-5 of the sum if all are off the same way, and some 16 u = 1e-6 as they fall."""
import numpy as np
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from oracle import tokens
from test_gpu_logits import BF16, F32, TOL, check_forward, cut, forward, make, near, teacher_of

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [F32, BF16])


@TYPES
@pytest.mark.parametrize("rows, n_v, parts, k", [(520, 1001, 1, 0), (520, 2503, 3, 0), (513, 9001, 2, 0), (512, 33001, 2, 0), (520, 2001, 9, 0), (600, 333, 20, 0),
                                                 (520, 1990, 1, 7), (520, 5003, 2, 64), (4100, 1203, 3, 20), (4096, 5003, 1, 33), (4097, 40, 20, 3)])
def test_forward(rows, n_v, parts, k, dtype):
    require_gpu()
    x, targets, _ = make(rows, n_v, dtype, 1)
    check_forward(x, targets, parts, k)


def test_equal_values_keep_their_order_in_one_wave():
    require_gpu()
    rows, n = 4100, 1301
    g = torch.Generator().manual_seed(1)
    ramp = torch.linspace(-20, 20, n)
    kinds = [torch.zeros(n), torch.randint(0, 2, (n,), generator=g).float(), ramp, ramp.flip(0), torch.where(torch.arange(n) % 3 == 0, -0.0, 0.0)]
    x = torch.stack([kinds[r % len(kinds)] for r in range(rows)])
    for dtype in (F32, BF16):
        y = x.to(dtype)
        _, (_, _, _, ids, _) = forward(y, torch.zeros(rows, dtype=torch.int32), 3, 40)
        want = np.argsort(-(y[:5].double().numpy() + 0.0), axis=1, kind="stable")[:, :40]
        assert np.array_equal(ids.cpu().numpy(), np.tile(want, (rows // 5, 1)))


@TYPES
def test_masks_infinities_and_nans(dtype):
    """A row that masks leave nothing of, one of the lowest value, one with a NaN, one with an infinity; the others are as without them."""
    require_gpu()
    for rows in (520, 4100):
        x, targets, _ = make(rows, 700, dtype, 6)
        targets[:4] = 5
        clean = forward(x, targets, 3, 9)[1]
        x[0], x[1], x[2, 17], x[3, 699] = -torch.inf, torch.finfo(dtype).min, torch.nan, torch.inf
        plan, got = forward(x, targets, 3, 9)
        logp, lse, entropy, ids, top = got
        for a, b in zip(clean, got):
            assert torch.equal(a[4:], b[4:])
        assert logp[0] == -torch.inf and lse[0] == -torch.inf and entropy[0] == 0
        near(logp[1:2], [-np.log(700.0)], TOL, "logp")
        near(entropy[1:2], [np.log(700.0)], TOL, "entropy")
        assert ids[1].tolist() == list(range(9))
        assert logp[2:4].isnan().all() and lse[2].isnan() and entropy[2:4].isnan().all()
        x_, ones = cut(x.cuda(), 3), torch.ones(rows, device="cuda")
        dx = [torch.full_like(t, 7.0) for t in x_]
        dd.distdl_logprob_bwd(plan, x_, targets.cuda(), lse, entropy, ones, ones, dx)
        dx = torch.cat(dx, 1)
        assert (dx[:2] == 0).all() and dx[2].isnan().all() and dx[4:].isfinite().all()


@TYPES
@pytest.mark.parametrize("rows, n_v, parts", [(520, 1001, 1), (520, 6001, 1), (513, 20011, 1), (512, 9001, 2), (520, 2001, 9), (600, 100, 33)])
def test_adjoint(rows, n_v, parts, dtype):
    require_gpu()
    x, targets, g = make(rows, n_v, dtype, 2)
    dlogp, dent = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    dlogp[2] = dent[2] = 0.0
    want = tokens.logprob_adjoint(x.double().numpy(), targets.numpy(), dlogp.double().numpy(), dent.double().numpy(), 0.8)
    plan, (_, lse, entropy, _, _) = forward(x, targets, parts, 0, 0.8)
    x_ = cut(x.cuda(), parts)
    dx = [torch.full_like(t, 7.0) for t in x_]
    args = targets.cuda(), lse, entropy, dlogp.cuda(), dent.cuda()
    dd.distdl_logprob_bwd(plan, x_, *args, dx, 0.8)
    got, size = torch.cat(dx, 1), np.abs(want).max(1, keepdims=True)
    near(got, want, 12 * TOL * size + 1e-7 + (2.0 ** -8 * np.abs(want) if dtype == BF16 else 0), "dx")
    dd.distdl_logprob_bwd(plan, x_, *args, x_, 0.8)  # in place
    assert torch.equal(torch.cat(x_, 1), got)


@TYPES
@pytest.mark.parametrize("rows, n_v, parts, k", [(520, 1001, 1, 17), (520, 1990, 3, 64), (513, 9001, 2, 17), (512, 36001, 1, 5), (512, 70001, 1, 64), (520, 9001, 9, 33), (600, 100, 33, 9),
                                                 (520, 1001, 1, 65), (513, 999, 2, 256), (512, 3001, 2, 300), (3, 5003, 2, 1024), (520, 1001, 1, 1000)])
@pytest.mark.parametrize("twice", [False, True])
def test_distill(rows, n_v, parts, k, twice, dtype):
    """Rows of one wave, rows that a workgroup keeps, and rows that it reads twice; places that come twice in one row, and in all."""
    require_gpu()
    x, _, g = make(rows, n_v, dtype, 4, masked=0.0)
    ids, teacher = teacher_of(rows, n_v, k, g)
    weight = torch.rand(rows, generator=g)
    ids[0, k // 2:] = -1
    ids[1] = ids[1, torch.arange(k) // 2]  # every place twice
    ids[2, 0], weight[2] = n_v, 0.0
    if twice:
        ids[:, -1] = ids[:, 0]
    ids[3 % rows] = -1
    want_loss, want = tokens.distill(x.double().numpy(), ids.numpy(), teacher.double().numpy(), weight.double().numpy(), 1.5)
    plan, x_ = dd.distdl_logits_plan_create(rows, n_v, parts, dtype), cut(x.cuda(), parts)
    loss, dx = torch.full((rows,), 7.0, device="cuda"), [torch.full_like(t, 7.0) for t in x_]
    args = ids.cuda(), teacher.cuda(), weight.cuda()
    dd.distdl_distill_fwd_bwd(plan, x_, *args, loss, dx, 1.5)
    near(loss, want_loss, 2 * TOL, "loss")
    got, size = torch.cat(dx, 1), np.abs(want).max(1, keepdims=True)
    near(got, want, TOL * size + 1e-7 + (2.0 ** -8 * np.abs(want) if dtype == BF16 else 0), "dx")
    alone = torch.full((rows,), 7.0, device="cuda")
    dd.distdl_distill_fwd_bwd(plan, x_, *args, alone, None, 1.5)
    near(alone, want_loss, 2 * TOL, "loss alone")
    dd.distdl_distill_fwd_bwd(plan, x_, *args, None, x_, 1.5)  # in place
    assert torch.equal(torch.cat(x_, 1), got)
