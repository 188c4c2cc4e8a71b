"""Rows of logits with numbers far from 0: masks that are numbers (-1e9, -1e10, -1e20), alone or beside entries of ordinary size, at several
temperatures; rows that are shifted as a whole.  Against the oracle in fp64.

Tolerances as in test_gpu_logits.py where what counts is of ordinary size (z is, at every temperature): differences of numbers near each other are exact.  An lse, or a log
probability of a masked entry, of size a is rounded a few times at that size: 2^-22 a.  A loss is a sum of t (log t - log p), and t is off by TOL of itself as p is there: where log p is
a mask's of size a, by TOL t a.  A gradient scale (p - t) is off by TOL scale (p + t), whatever is left of it."""
import numpy as np
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from oracle import tokens
from test_gpu_logits import BF16, F32, TOL, cut, forward, near

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [F32, BF16])
MASKS = pytest.mark.parametrize("mask", [-1e9, -1e10, -1e20])
SIZE = 2.0 ** -22
# rows, entries, workers: cut rows, a workgroup's, a wave's, tiny parts
SHAPES = [(7, 20011, 3), (2, 90000, 1), (520, 9001, 2), (520, 1203, 3), (600, 100, 33)]


def masked(rows, n_v, dtype, mask, temperature, seed=0):
    """Seven kinds of rows by turns: nothing but the mask, one entry left, a masked front, a masked end, a masked middle, every other entry masked, no mask."""
    g = torch.Generator().manual_seed(seed)
    x = (3 * temperature * torch.randn(rows, n_v, generator=g)).to(dtype)
    at = torch.arange(n_v)
    kinds = [at >= 0, at != n_v // 3, at < n_v * 3 // 4, at >= n_v // 4, (at >= n_v // 5) & (at < n_v - 2), at % 2 == 0, at < 0]
    for r in range(rows):
        x[r, kinds[r % 7]] = mask
    targets = torch.randint(0, n_v, (rows,), generator=g, dtype=torch.int32)
    if rows > 1:
        targets[1] = n_v // 3
    return x, targets, g


def check_forward(x, targets, parts, k, temperature):
    _, (logp, lse, entropy, ids, top) = forward(x, targets, parts, k, temperature)
    want = tokens.logprob_forward(x.double().numpy(), targets.numpy(), k, temperature)
    for got, w, what in ((logp, want[0], "logp"), (lse, want[1], "lse"), (entropy, want[2], "entropy")) + (((top, want[4], "top"),) if k else ()):
        near(got, w, TOL + SIZE * np.abs(w), what)
    if k:
        assert np.array_equal(ids.cpu().numpy(), want[3])


@TYPES
@MASKS
@pytest.mark.parametrize("rows, n_v, parts", SHAPES)
def test_masks_that_are_numbers(rows, n_v, parts, mask, dtype):
    require_gpu()
    for temperature in (1.0, 0.3, 0.1, 2.0):
        x, targets, _ = masked(rows, n_v, dtype, mask, temperature)
        for k in (0, 9):
            check_forward(x, targets, parts, k, temperature)


@pytest.mark.parametrize("shift", [726817.0, -726817.0, 1e6, -1e6, 1e7])
@pytest.mark.parametrize("rows, n_v, parts", SHAPES)
def test_shifted_rows(rows, n_v, parts, shift):
    """A row that is shifted has the same log probabilities.  In units of log 2 the first shifts are 2^20, so some entries are below it and some above."""
    require_gpu()
    g = torch.Generator().manual_seed(1)
    x = shift + 4 * torch.randn(rows, n_v, generator=g)
    check_forward(x, torch.randint(0, n_v, (rows,), generator=g, dtype=torch.int32), parts, 9, 1.0)


@pytest.mark.parametrize("temperature", [1e-6, 1e-3, 1e6])
def test_all_temperatures(temperature):
    """Logits of 5000 at the lowest temperature are 7e9 in units of log 2; neighbouring numbers are so far apart there that the largest has everything."""
    require_gpu()
    for rows in (5, 520):
        g = torch.Generator().manual_seed(2)
        x = 5000 + torch.randn(rows, 3001, generator=g)
        x[1], x[2, :2000] = 5000.0, 5000.0
        check_forward(x, torch.randint(0, 3001, (rows,), generator=g, dtype=torch.int32), 2, 5, temperature)


@TYPES
@MASKS
@pytest.mark.parametrize("rows, n_v, parts, k", [(7, 20011, 3, 9), (520, 1001, 1, 9), (520, 9001, 2, 9), (512, 70001, 1, 9), (520, 1203, 3, 70), (600, 100, 33, 9)])
def test_distillation_of_a_masked_student(rows, n_v, parts, k, mask, dtype):
    """One wave's rows, kept ones, ones that are read twice and cut ones.  The teacher has places that the mask leaves, where it leaves enough."""
    require_gpu()
    for temperature in (1.0, 0.1):
        x, _, g = masked(rows, n_v, dtype, mask, temperature, 3)
        order = torch.argsort(-x.float(), dim=1, stable=True)
        ids = torch.stack([o[torch.randperm(k + 15, generator=g)[:k]] for o in order]).to(torch.int32)
        ids[1], ids[1, 0] = -1, n_v // 3
        teacher, weight = 2 * temperature * torch.randn(rows, k, generator=g), 0.5 + torch.rand(rows, generator=g)
        want_loss, want = tokens.distill(x.double().numpy(), ids.numpy(), teacher.double().numpy(), weight.double().numpy(), temperature)
        plan, x_ = dd.distdl_logits_plan_create(rows, n_v, parts, dtype), cut(x.cuda(), parts)
        loss, dx = torch.full((rows,), 7.0, device="cuda"), [torch.full_like(t, 7.0) for t in x_]
        dd.distdl_distill_fwd_bwd(plan, x_, ids.cuda(), teacher.cuda(), weight.cuda(), loss, dx, temperature)
        near(loss, want_loss, 2 * TOL + TOL * np.abs(want_loss), "loss")
        scale = weight.double().numpy()[:, None] / temperature
        p = np.exp(tokens.log_softmax(x.double().numpy(), temperature)[0])
        size = p + np.abs(p - want / scale)  # p + t
        near(torch.cat(dx, 1), want, TOL * scale * size + 1e-12 + (2.0 ** -8 * np.abs(want) if dtype == BF16 else 0), "dx")


@TYPES
@pytest.mark.parametrize("rows, n_v, parts, k", [(9, 20011, 3, 9), (520, 1001, 1, 9), (520, 9001, 2, 9), (512, 36001, 1, 9), (520, 1203, 3, 70), (600, 100, 33, 9)])
def test_distillation_from_a_teacher_of_large_numbers(rows, n_v, parts, k, dtype):
    """By turns: the lowest number at all places, at place 0 again and again (padding), one place with it, with -1e10, 1e10 and the largest number, equal large ones, ordinary ones
    beside the lowest, ordinary ones.  One place with any finite logit is the cross entropy."""
    require_gpu()
    low = torch.finfo(F32).min
    for temperature in (1.0, 0.25, 4.0):
        g = torch.Generator().manual_seed(5)
        x = (3 * temperature * torch.randn(rows, n_v, generator=g)).to(dtype)
        ids = torch.stack([torch.randperm(n_v, generator=g)[:k] for _ in range(rows)]).to(torch.int32)
        teacher, weight = 2 * temperature * torch.randn(rows, k, generator=g), 0.5 + torch.rand(rows, generator=g)
        for r in range(rows):
            kind = r % 9
            if kind in (0, 1):
                teacher[r] = low
                ids[r] = ids[r] if kind == 0 else 0
            elif kind < 6:
                ids[r, 1:], teacher[r, 0] = -1, (low, -1e10, 1e10, -low)[kind - 2]
            elif kind == 6:
                teacher[r] = 1e20
            elif kind == 7:
                teacher[r, ::2] = low
        weight[1] = 0.0  # (its loss is a number too)
        want_loss, want = tokens.distill(x.double().numpy(), ids.numpy(), teacher.double().numpy(), weight.double().numpy(), temperature)
        plan, x_ = dd.distdl_logits_plan_create(rows, n_v, parts, dtype), cut(x.cuda(), parts)
        loss, dx = torch.full((rows,), 7.0, device="cuda"), [torch.full_like(t, 7.0) for t in x_]
        dd.distdl_distill_fwd_bwd(plan, x_, ids.cuda(), teacher.cuda(), weight.cuda(), loss, dx, temperature)
        near(loss, want_loss, 2 * TOL, "loss")
        scale = weight.double().numpy()[:, None] / temperature
        p = np.exp(tokens.log_softmax(x.double().numpy(), temperature)[0])
        size = p * scale + np.abs(p * scale - want)  # of p and t
        near(torch.cat(dx, 1), want, TOL * size + 1e-12 + (2.0 ** -8 * np.abs(want) if dtype == BF16 else 0), "dx")
        log_p = tokens.log_softmax(x.double().numpy(), temperature)[0]
        alone = [r for r in range(rows) if 2 <= r % 9 < 6]
        near(loss[alone], [-log_p[r, ids[r, 0]] for r in alone], 2 * TOL, "cross entropy")


@pytest.mark.parametrize("shift", [0.0, 1e3, -1e5, 5e5, 7e5, 1e6])
@pytest.mark.parametrize("rows, n_v, parts, k", [(7, 20011, 3, 9), (520, 1001, 1, 9), (520, 9001, 2, 9), (512, 36001, 1, 9)])
def test_gradients_of_shifted_rows(rows, n_v, parts, k, shift):
    """x is rounded once it is shifted, the oracle has it as it is.  What a shift would cost were it in a number of its size: 2^-24 of 1e6 / ln 2, 9 % of p."""
    require_gpu()
    g = torch.Generator().manual_seed(6)
    x = shift + 3 * torch.randn(rows, n_v, generator=g)
    ids = torch.stack([torch.randperm(n_v, generator=g)[:k] for _ in range(rows)]).to(torch.int32)
    teacher, weight = 2 * torch.randn(rows, k, generator=g), 0.5 + torch.rand(rows, generator=g)
    want_loss, want = tokens.distill(x.double().numpy(), ids.numpy(), teacher.double().numpy(), weight.double().numpy())
    plan, x_ = dd.distdl_logits_plan_create(rows, n_v, parts, F32), cut(x.cuda(), parts)
    loss, dx = torch.full((rows,), 7.0, device="cuda"), [torch.full_like(t, 7.0) for t in x_]
    dd.distdl_distill_fwd_bwd(plan, x_, ids.cuda(), teacher.cuda(), weight.cuda(), loss, dx)
    near(loss, want_loss, 2 * TOL, "loss")
    scale = weight.double().numpy()[:, None]
    p = np.exp(tokens.log_softmax(x.double().numpy())[0])
    size = p * scale + np.abs(p * scale - want)
    near(torch.cat(dx, 1), want, TOL * size + 1e-12, "dx")


def test_gradients_are_as_near_as_the_rounding_of_differences():
    """Rows of ordinary logits, |z - lse| up to 25, 36 in units of log 2.  p = exp2(d) with d = (x c - m c) - log2 s: its two differences are rounded by up to 36 u each, half of that
    as a rule, log2 s and exp2 by u of 12 and of p: less than 36 u ln 2 = 1.5e-6 of p by root mean square, and with most of the sum of squares in entries with d above -20 some 4e-7."""
    require_gpu()
    g = torch.Generator().manual_seed(7)
    x = 3 * torch.randn(64, 10007, generator=g) + 11
    ids, teacher = torch.randint(0, 10007, (64, 17), generator=g, dtype=torch.int32), torch.randn(64, 17, generator=g)
    want = tokens.distill(x.double().numpy(), ids.numpy(), teacher.double().numpy(), np.ones(64))[1]
    plan, x_ = dd.distdl_logits_plan_create(64, 10007, 3, F32), cut(x.cuda(), 3)
    dx = [torch.empty_like(t) for t in x_]
    dd.distdl_distill_fwd_bwd(plan, x_, ids.cuda(), teacher.cuda(), None, None, dx)
    got = torch.cat(dx, 1).double().cpu().numpy()
    rest = np.ones(got.shape, bool)  # (without the teacher's places, which are computed for themselves)
    np.put_along_axis(rest, ids.numpy(), False, 1)
    assert np.linalg.norm((got - want)[rest]) <= 4e-7 * np.linalg.norm(want[rest])


@TYPES
@pytest.mark.parametrize("rows, n_v, parts", [(7, 20011, 3), (520, 9001, 2), (520, 1203, 3), (600, 100, 33)])
def test_log_probabilities_of_the_lowest_value(rows, n_v, parts, dtype):
    """Masks of the type's lowest value are numbers, and so are their log probabilities: -3.4e38, where it is in the range of 32 bits over the temperature."""
    require_gpu()
    for temperature in (1.0, 1.7):
        x, _, g = masked(rows, n_v, dtype, torch.finfo(dtype).min, temperature, 8)
        targets = torch.randint(0, n_v, (rows,), generator=g, dtype=torch.int32)
        for r in range(rows):
            if r % 7 in (1, 2, 5):
                targets[r] = 0  # masked
        check_forward(x, targets, parts, 9, temperature)
        ids = targets[:, None].repeat(1, 2).contiguous()
        ids[:, 1] = (ids[:, 0] + 1) % n_v
        teacher = torch.tensor([[0.0, 1.0]]).repeat(rows, 1).contiguous()
        loss = torch.full((rows,), 7.0, device="cuda")
        plan, x_ = dd.distdl_logits_plan_create(rows, n_v, parts, dtype), cut(x.cuda(), parts)
        dd.distdl_distill_fwd_bwd(plan, x_, ids.cuda(), teacher.cuda(), None, loss, None, temperature)
        want = tokens.distill(x.double().numpy(), ids.numpy(), teacher.double().numpy(), np.ones(rows), temperature)[0]
        near(loss, want, 2 * TOL + TOL * np.abs(want), "loss")
        dx = [torch.full_like(t, 7.0) for t in x_]
        again = torch.full((rows,), 7.0, device="cuda")
        dd.distdl_distill_fwd_bwd(plan, x_, ids.cuda(), teacher.cuda(), None, again, dx, temperature)
        near(again, want, 2 * TOL + TOL * np.abs(want), "loss beside a gradient")


def check_adjoint(x, targets, parts, temperature, g):
    """p is off by TOL of itself and log p + H by 2 TOL; in place gives the same bits."""
    rows, dtype = x.shape[0], x.dtype
    dlogp, dent = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    plan, (_, lse, entropy, _, _) = forward(x, targets, parts, 0, temperature)
    n, w, e = x.double().numpy(), dlogp.double().numpy()[:, None], dent.double().numpy()[:, None]
    log_p = tokens.log_softmax(n, temperature)[0]
    p, live = np.exp(log_p), ((targets >= 0) & (targets < x.shape[1])).numpy()
    hit = np.zeros(n.shape)
    hit[live, targets.numpy()[live]] = 1
    for what in ("logp", "entropy", "both"):
        with_w, with_e = w * (what != "entropy") * live[:, None], e * (what != "logp")
        want = tokens.logprob_adjoint(n, targets.numpy(), with_w[:, 0], with_e[:, 0], temperature)
        size = np.abs(with_w) * (hit + p) + np.abs(with_e) * p * (np.maximum(np.abs(log_p), -200) + np.log(x.shape[1]) + 2)
        x_ = cut(x.cuda(), parts)
        args = (targets.cuda(), lse, entropy if what != "logp" else None, dlogp.cuda() if what != "entropy" else None, dent.cuda() if what != "logp" else None)
        dx = [torch.full_like(t, 7.0) for t in x_]
        dd.distdl_logprob_bwd(plan, x_, *args, dx, temperature)
        got = torch.cat(dx, 1)
        near(got, want, TOL * size / temperature + 1e-12 + (2.0 ** -8 * np.abs(want) if dtype == BF16 else 0), what)
        dd.distdl_logprob_bwd(plan, x_, *args, x_, temperature)
        assert torch.equal(torch.cat(x_, 1), got)


@TYPES
@MASKS
@pytest.mark.parametrize("rows, n_v, parts", [(7, 20011, 3), (2, 70001, 1), (520, 3001, 2), (520, 9001, 1), (600, 100, 33)])
def test_adjoint_of_masks_that_are_numbers(rows, n_v, parts, mask, dtype):
    """A row of nothing but the mask is an even one, though its lse cannot hold how many entries it has."""
    require_gpu()
    for temperature in (1.0, 0.3):
        x, targets, g = masked(rows, n_v, dtype, mask, temperature, 9)
        check_adjoint(x, targets, parts, temperature, g)


@pytest.mark.parametrize("shift", [200.0, -300.0, 5e3, -1e5, 1e6, 1e7])
@pytest.mark.parametrize("rows, n_v, parts", [(7, 20011, 3), (520, 1203, 3), (520, 9001, 1)])
def test_adjoint_of_shifted_rows(rows, n_v, parts, shift):
    require_gpu()
    g = torch.Generator().manual_seed(10)
    x = shift + 3 * torch.randn(rows, n_v, generator=g)
    targets = torch.randint(-1, n_v, (rows,), generator=g, dtype=torch.int32)
    check_adjoint(x, targets, parts, 1.0, g)


@pytest.mark.parametrize("dtype, bits", [(F32, 0x7f800001), (F32, -1), (BF16, 0x7f81), (BF16, -1)])
@pytest.mark.parametrize("rows", [3, 520, 4100])
def test_nans_of_all_kinds_are_no_alternatives(rows, dtype, bits):
    """Signalling NaNs too, beside the best entries: a maximum of one and a number is the NaN.  Half of the rows have none."""
    require_gpu()
    g = torch.Generator().manual_seed(11)
    x = torch.randn(rows, 3001, generator=g).to(dtype)
    top = x.float().argsort(dim=1, descending=True, stable=True)[:, :8]
    clean = x.clone()
    raw = x.view(torch.int32 if dtype == F32 else torch.int16)
    for r in range(0, rows, 2):
        at = int(top[r, r // 2 % 8])
        for j in range(at // 8 * 8, min(at // 8 * 8 + 8, 3001)):
            if j not in top[r].tolist() and (j + r // 2) % 2:
                raw[r, j] = bits
    _, (_, lse, _, ids, _) = forward(x, torch.zeros(rows, dtype=torch.int32), 1, 8)
    want = torch.nan_to_num(x.float(), nan=-torch.inf).argsort(dim=1, descending=True, stable=True)[:, :8]
    assert torch.equal(ids.cpu().long(), want)
    assert torch.equal(lse.isnan().cpu(), x.float().isnan().any(1))
    assert torch.equal(x[1::2], clean[1::2])
