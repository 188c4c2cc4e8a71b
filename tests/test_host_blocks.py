"""Refusals of the operators of gated recurrent blocks: no device is needed, nothing is launched, outputs stay as they were."""
import ctypes as C

import pytest
import torch

import paper_2006_03108_amd as dd

INVALID, NULL, UNSUPPORTED, EMPTY = -1, -2, -3, -4
BF16, F32 = torch.bfloat16, torch.float32


def code(f, *a, **k):
    with pytest.raises(dd.DistdlError) as e:
        f(*a, **k)
    assert str(e.value)
    return e.value.code


def test_plans():
    assert code(dd.distdl_rmsnorm_plan_create, -1, 8, 1, 1e-6) == INVALID
    assert code(dd.distdl_rmsnorm_plan_create, 4, 0, 1, 1e-6) == INVALID
    assert code(dd.distdl_rmsnorm_plan_create, 4, 3, 4, 1e-6) == EMPTY
    assert code(dd.distdl_rmsnorm_plan_create, 4, 8, 1, -1.0) == INVALID
    assert code(dd.distdl_rmsnorm_plan_create, 4, 8, 1, float("nan")) == INVALID
    assert code(dd.distdl_rmsnorm_plan_create, 4, 8, 1, 1e-6, torch.float16) == UNSUPPORTED
    assert code(dd.distdl_rmsnorm_plan_create, 1 << 40, 8, 1, 1e-6) == UNSUPPORTED
    assert code(dd.distdl_linear8_plan_create, 0, 8, 8, 1, 1) == INVALID
    assert code(dd.distdl_linear8_plan_create, 4, 8, 8, 9, 1) == EMPTY
    assert code(dd.distdl_linear8_plan_create, 4, 1 << 31, 8, 1, 1) == UNSUPPORTED
    assert code(dd.distdl_scan_plan_create, 0, 4, 4, 1, "given") == INVALID
    assert code(dd.distdl_scan_plan_create, 1, 4, 4, 5, "given") == EMPTY
    assert code(dd.distdl_scan_plan_create, 1, 4, 4, 1, "tanh") == UNSUPPORTED
    assert code(dd.distdl_scan_plan_create, 1, 1 << 31, 4, 1, "given") == UNSUPPORTED
    assert code(dd.distdl_adamw_plan_create, []) == INVALID
    assert code(dd.distdl_adamw_plan_create, [4, -1]) == INVALID
    assert code(dd.distdl_adamw_plan_create, [4], torch.float16) == UNSUPPORTED


def test_tensors_are_held_against_the_plan():
    """Wrong type, size, layout, number and place, before anything is enqueued."""
    plan = dd.distdl_rmsnorm_plan_create(4, 8, 1, 1e-6, F32)
    g, y = [torch.ones(8)], [torch.full((4, 8), 3.0)]
    for x in (torch.zeros(4, 7), torch.zeros(4, 8, dtype=BF16), torch.zeros(8, 4).t(), torch.zeros(4, 8)):  # (the last lies on the host)
        assert code(dd.distdl_rmsnorm_fwd, plan, [x], None, g, None, y, None, None, None) == INVALID
    assert code(dd.distdl_rmsnorm_fwd, plan, [], None, g, None, y, None, None, None) == INVALID
    assert (y[0] == 3.0).all()
    plan = dd.distdl_scan_plan_create(2, 6, 5, 2, "sigmoid", F32)
    three = [torch.zeros(2, 3, 5)] * 2
    assert code(dd.distdl_scan_fwd, plan, three, three, None, None, three, None) == INVALID
    assert code(dd.distdl_scan_fwd, plan, three[:1], three, None, None, three, None) == INVALID
    assert code(dd.distdl_scan_step, torch.zeros(2, 5), torch.zeros(2, 5), torch.zeros(2, 6), None, torch.zeros(2, 5), "given") == INVALID
    assert code(dd.distdl_quant8, [torch.zeros(3)], None, None, None, None) == INVALID
    assert code(dd.distdl_quant8, [], [], [], None, None) == INVALID
    plan = dd.distdl_adamw_plan_create([4], F32, states8=True)
    four = [torch.zeros(4)]
    assert code(dd.distdl_adamw_step, plan, four, four, four, four, lr=1e-3, step=1) == NULL
    assert code(dd.distdl_adamw_step, plan, four, four, four, four, four, four, lr=1e-3, step=1) == INVALID


KEPT = []


def handle(plan):
    """Its handle; the plan is kept for as long."""
    KEPT.append(plan)
    return plan.handle


def some(*addresses):
    return (C.c_void_p * len(addresses))(*addresses)


def test_entry_points():
    """The C boundary itself: pointers are numbers that nobody follows."""
    ok, odd = some(0x10000), some(0x10001)
    norm = handle(dd.distdl_rmsnorm_plan_create(4, 8, 1, 1e-6, F32))
    fwd = dd.lib.distdl_rmsnorm_fwd
    assert fwd(None, ok, None, ok, None, ok, None, None, None, None) == NULL
    assert fwd(norm, ok, None, ok, None, None, None, None, None, None) == NULL  # no output
    assert fwd(norm, ok, None, ok, None, None, ok, None, None, None) == NULL    # codes without scales
    assert fwd(norm, ok, None, ok, None, some(None), None, None, None, None) == NULL
    assert fwd(norm, odd, None, ok, None, ok, None, None, None, None) == INVALID
    assert fwd(norm, ok, None, ok, None, ok, None, None, 0x10002, None) == INVALID
    assert dd.lib.distdl_rmsnorm_bwd(norm, ok, ok, None, ok, None, ok, ok, None) == NULL
    one = (C.c_int64 * 1)(5)
    quant = dd.lib.distdl_quant8
    assert quant(None, one, one, 1, 0, ok, ok, None, None, 0, None) == NULL
    assert quant(ok, one, one, 1, 0, ok, None, None, None, 0, None) == NULL
    assert quant(ok, one, one, 1, 0, None, None, None, None, 0, None) == NULL
    assert quant(ok, one, one, 0, 0, ok, ok, None, None, 0, None) == INVALID
    assert quant(ok, one, (C.c_int64 * 1)(-1), 1, 0, ok, ok, None, None, 0, None) == INVALID
    assert quant(odd, one, one, 1, 0, ok, ok, None, None, 0, None) == INVALID
    assert quant(ok, one, one, 1, 0, ok, ok, None, None, 7, None) == UNSUPPORTED
    layer = handle(dd.distdl_linear8_plan_create(4, 8, 8, 1, 1, BF16))
    assert dd.lib.distdl_linear8_fwd(layer, ok, ok, ok, ok, odd, None) == INVALID
    assert dd.lib.distdl_linear8_fwd(layer, ok, ok, ok, None, ok, None) == NULL
    assert dd.lib.distdl_linear8_bwd_x(layer, ok, ok, ok, some(None), ok, None) == NULL
    assert dd.lib.distdl_linear8_bwd_w(layer, ok, ok, ok, ok, odd, None) == INVALID
    scan = handle(dd.distdl_scan_plan_create(1, 4, 4, 1, "sigmoid", BF16))
    assert dd.lib.distdl_scan_fwd(scan, ok, None, None, None, ok, None, None) == NULL
    assert dd.lib.distdl_scan_fwd(scan, ok, ok, 0x10002, None, ok, None, None) == INVALID
    assert dd.lib.distdl_scan_bwd(scan, ok, None, ok, None, None, ok, None, ok, ok, None, None) == NULL  # sigmoid gates read x
    step = dd.lib.distdl_scan_step
    assert step(0x1000, 0x1000, 0x1000, 3, None, 0x1000, 4, 8, 0, 0, None) == INVALID  # four rows, three states
    assert step(0x1000, 0x1000, None, 4, None, 0x1000, 4, 8, 0, 0, None) == NULL
    assert step(0x1000, 0x1000, 0x1000, 4, None, 0x1000, 4, 0, 0, 0, None) == INVALID
    assert step(0x1000, 0x1000, 0x1000, 4, None, 0x1000, 4, 8, 2, 0, None) == UNSUPPORTED
    assert step(None, None, None, 0, None, None, 0, 8, 0, 0, None) == 0  # no rows
    adam = handle(dd.distdl_adamw_plan_create([4], F32))
    good = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, step=1)
    update = lambda p=ok, **k: dd.lib.distdl_adamw_step(adam, p, ok, ok, ok, None, None, None, C.byref(dd.AdamwArgs(**{**good, **k})), None)  # noqa: E731
    for bad in (dict(lr=-1.0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(weight_decay=float("inf")),
                dict(weight_decay=-0.1), dict(step=0), dict(step_dev=0x10004), dict(gscale_dev=0x10002)):
        assert update(**bad) == INVALID, bad
    assert update(some(None)) == NULL and update(odd) == INVALID
    assert dd.lib.distdl_adamw_step(adam, ok, ok, ok, ok, None, None, None, None, None) == NULL


def test_many_workers_and_nothing_to_do():
    """The host code of calls with more workers than travel with a launch, up to the first device call, which fails here."""
    if torch.cuda.is_available():
        pytest.skip("meant for a machine without a device")
    for P in (8, 9, 16, 17, 70):
        many = some(*[0x10000 * (i + 1) for i in range(P * 2)])
        norm = handle(dd.distdl_rmsnorm_plan_create(4, 300, P, 1e-6, F32))
        assert dd.lib.distdl_rmsnorm_fwd(norm, many, many, many, many, many, many, many, None, None) in (-6, -7)
        layer = handle(dd.distdl_linear8_plan_create(4, 300, 300, P, 2, BF16))
        assert dd.lib.distdl_linear8_fwd(layer, many, many, many, many, many, None) in (-6, -7)
        scan = handle(dd.distdl_scan_plan_create(2, 400, 9, P, "given", F32))
        assert dd.lib.distdl_scan_fwd(scan, many, many, None, None, many, None, None) in (-6, -7)
        sizes = (C.c_int64 * P)(*[5] * P)
        assert dd.lib.distdl_quant8(many, sizes, sizes, P, 0, many, many, None, None, 0, None) in (-6, -7)
    # empty tensors have no address; a plan of none has nothing to do
    none = some(None)
    empty = handle(dd.distdl_adamw_plan_create([0], F32))
    args = dd.AdamwArgs(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, step=1)
    assert dd.lib.distdl_adamw_step(empty, none, none, none, none, None, None, None, C.byref(args), None) == 0
    zero = (C.c_int64 * 1)(0)
    assert dd.lib.distdl_quant8(none, zero, zero, 1, 0, none, none, None, None, 0, None) == 0
    norm = handle(dd.distdl_rmsnorm_plan_create(0, 8, 1, 1e-6, F32))
    assert dd.lib.distdl_rmsnorm_fwd(norm, none, None, some(0x1000), None, none, None, None, None, None) == 0
