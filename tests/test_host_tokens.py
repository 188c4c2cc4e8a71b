"""Refusals of the operators of a model of tokens: no device is needed, nothing is launched, outputs stay as they were."""
import ctypes as C

import pytest
import torch

import paper_2006_03108_amd as dd

INVALID, NULL, UNSUPPORTED, EMPTY = -1, -2, -3, -4
BF16, F32 = torch.bfloat16, torch.float32
KEPT = []


def code(f, *a, **k):
    with pytest.raises(dd.DistdlError) as e:
        f(*a, **k)
    assert str(e.value)
    return e.value.code


def handle(plan):
    """Its handle; the plan is kept for as long."""
    KEPT.append(plan)
    return plan.handle


def some(*addresses):
    return (C.c_void_p * len(addresses))(*addresses)


def test_plans():
    assert code(dd.distdl_delta_plan_create, 0, 4, 2, 1, 8, 8, 1, 1.0) == INVALID
    assert code(dd.distdl_delta_plan_create, 1, 4, 3, 2, 8, 8, 1, 1.0) == INVALID  # heads that keys do not divide
    assert code(dd.distdl_delta_plan_create, 1, 4, 2, 1, 0, 8, 1, 1.0) == INVALID
    assert code(dd.distdl_delta_plan_create, 1, 4, 2, 1, 8, 8, 1, float("nan")) == INVALID
    assert code(dd.distdl_delta_plan_create, 1, 4, 2, 1, 8, 8, 5, 1.0) == EMPTY
    assert code(dd.distdl_delta_plan_create, 1, 4, 2, 1, 129, 8, 1, 1.0) == UNSUPPORTED
    assert code(dd.distdl_delta_plan_create, 1, 1 << 31, 2, 1, 8, 8, 1, 1.0) == UNSUPPORTED
    assert code(dd.distdl_delta_plan_create, 1, 4, 1 << 12, 1, 8, 1 << 12, 1, 1.0) == UNSUPPORTED
    assert code(dd.distdl_delta_plan_create, 1, 4, 1 << 16, 1 << 16, 128, 1, 1, 1.0) == UNSUPPORTED
    assert code(dd.distdl_delta_plan_create, 1 << 19, 1, 16, 1, 1, 16, 1, 1.0) == UNSUPPORTED  # 2^32 threads of a launch
    assert code(dd.distdl_delta_plan_create, 1, 4, 2, 1, 8, 8, 1, 1.0, torch.float16) == UNSUPPORTED
    assert code(dd.distdl_logits_plan_create, -1, 8, 1) == INVALID
    assert code(dd.distdl_logits_plan_create, 4, 0, 1) == INVALID
    assert code(dd.distdl_logits_plan_create, 4, 3, 4) == EMPTY
    assert code(dd.distdl_logits_plan_create, 4, 1 << 30, 1) == UNSUPPORTED
    assert code(dd.distdl_logits_plan_create, 1 << 40, 8, 1) == UNSUPPORTED
    assert code(dd.distdl_logits_plan_create, 4, 8, 1, torch.float16) == UNSUPPORTED


def test_tensors_are_held_against_the_plan():
    """Wrong type, size, layout, number and place, before anything is enqueued."""
    plan = dd.distdl_logits_plan_create(4, 8, 2, F32)
    rows = torch.zeros(4)
    for x in ([torch.zeros(4, 4)] * 2, [torch.zeros(4, 4)], [torch.zeros(4, 5)] * 2, [torch.zeros(4, 4, dtype=BF16)] * 2, [torch.zeros(4, 4).t()] * 2):
        assert code(dd.distdl_logprob_fwd, plan, x, None, None, rows, None) == INVALID  # (the first lies on the host)
    x = [torch.zeros(4, 4)] * 2
    ids, top = torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 2)
    assert code(dd.distdl_logprob_fwd, plan, x, None, None, rows, None, ids, top) == INVALID  # of different widths
    assert code(dd.distdl_logprob_fwd, plan, x, None, None, rows, None, ids[:3], None) == INVALID
    assert code(dd.distdl_distill_fwd_bwd, plan, x, ids, top, None, rows, None) == INVALID
    assert (rows == 0).all()
    plan = dd.distdl_delta_plan_create(2, 6, 4, 2, 5, 3, 2, 1.0, F32)
    key, value, gate = [torch.zeros(2, 3, 2, 5)] * 2, [torch.zeros(2, 3, 4, 3)] * 2, [torch.zeros(2, 3, 4)] * 2
    assert code(dd.distdl_delta_fwd, plan, key, key, value, gate, gate, None, None, value, None) == INVALID
    assert code(dd.distdl_delta_fwd, plan, value, key, value, gate, gate, None, None, value, None) == INVALID
    assert code(dd.distdl_delta_fwd, plan, key[:1], key, value, gate, gate, None, None, value, None) == INVALID
    q, v, state = torch.zeros(2, 2, 5), torch.zeros(2, 4, 3), torch.zeros(2, 4, 5, 3)
    for wrong in ((q[0], v, state), (q, v[:1], state), (q, v, state[:, :3]), (q, v, state[..., :2]), (q, v, state)):
        assert code(dd.distdl_delta_step, wrong[0], wrong[0], wrong[1], None, torch.zeros(2, 4), wrong[2], None, wrong[1], 1.0) == INVALID


def test_logits_entry_points():
    """The C boundary itself: pointers are numbers that nobody follows."""
    ok, odd, none = some(0x10000), some(0x10002), some(None)
    f32 = handle(dd.distdl_logits_plan_create(4, 100, 1, F32))
    fwd, bwd, distill = dd.lib.distdl_logprob_fwd, dd.lib.distdl_logprob_bwd, dd.lib.distdl_distill_fwd_bwd
    p = 0x20000
    assert fwd(None, ok, p, p, p, p, None, None, 0, 1.0, None) == NULL
    assert fwd(f32, None, p, p, p, p, None, None, 0, 1.0, None) == NULL
    assert fwd(f32, none, p, p, p, p, None, None, 0, 1.0, None) == NULL
    assert fwd(f32, ok, None, p, p, p, None, None, 0, 1.0, None) == NULL    # log probabilities without targets
    assert fwd(f32, ok, p, None, None, None, None, None, 0, 1.0, None) == NULL  # no output
    assert fwd(f32, ok, p, None, p, None, None, None, 3, 1.0, None) == NULL    # alternatives without a place
    assert fwd(f32, ok, p, None, p, None, p, p, 0, 1.0, None) == INVALID
    assert fwd(f32, ok, p, None, p, None, p, p, -1, 1.0, None) == INVALID
    assert fwd(f32, ok, p, None, p, None, p, p, 101, 1.0, None) == INVALID
    assert fwd(f32, ok, p, None, p, None, p, p, 65, 1.0, None) == UNSUPPORTED
    assert fwd(f32, odd, p, None, p, None, None, None, 0, 1.0, None) == INVALID
    assert fwd(f32, ok, p, None, p + 2, None, None, None, 0, 1.0, None) == INVALID
    for temperature in (0.0, -1.0, 1e-7, 1e7, float("nan"), float("inf")):
        assert fwd(f32, ok, p, None, p, None, None, None, 0, temperature, None) == INVALID
    assert bwd(f32, ok, p, None, p, p, p, ok, 1.0, None) == NULL               # no lse
    assert bwd(f32, ok, p, p, p, None, None, ok, 1.0, None) == NULL            # no gradient
    assert bwd(f32, ok, None, p, p, p, None, ok, 1.0, None) == NULL            # dlogp without targets
    assert bwd(f32, ok, p, p, None, None, p, ok, 1.0, None) == NULL            # dentropy without the entropy
    assert bwd(f32, ok, p, p, p, p, p, None, 1.0, None) == NULL
    assert bwd(f32, ok, p, p, p, p, p, none, 1.0, None) == NULL
    assert bwd(f32, ok, p, p, p, p, p, odd, 1.0, None) == INVALID
    assert distill(f32, ok, p, p, 0, p, p, ok, 1.0, None) == INVALID
    assert distill(f32, ok, p, p, 1025, p, p, ok, 1.0, None) == UNSUPPORTED
    assert distill(f32, ok, None, p, 4, p, p, ok, 1.0, None) == NULL
    assert distill(f32, ok, p, None, 4, p, p, ok, 1.0, None) == NULL
    assert distill(f32, ok, p, p, 4, p, None, None, 1.0, None) == NULL
    assert distill(f32, ok, p, p, 4, p, p, ok, 0.0, None) == INVALID
    assert distill(f32, ok, p + 1, p, 4, p, p, ok, 1.0, None) == INVALID
    empty = handle(dd.distdl_logits_plan_create(0, 100, 1, F32))
    assert fwd(empty, none, None, None, p, None, None, None, 0, 1.0, None) == 0
    assert bwd(empty, none, None, None, None, None, None, none, 1.0, None) == 0
    assert distill(empty, none, None, None, 3, None, None, none, 1.0, None) == 0


def test_delta_entry_points():
    ok, odd, none, p = some(0x10000), some(0x10002), some(None), 0x20000
    plan = handle(dd.distdl_delta_plan_create(1, 4, 2, 1, 8, 8, 1, 1.0, F32))
    fwd, bwd, step = dd.lib.distdl_delta_fwd, dd.lib.distdl_delta_bwd, dd.lib.distdl_delta_step
    good = [plan, ok, ok, ok, ok, ok, None, None, ok, None, None]
    for i in (0, 1, 2, 3, 5, 8):
        assert fwd(*good[:i], None, *good[i + 1:]) == NULL
    for i in (1, 2, 3, 4, 5, 8):
        assert fwd(*good[:i], none, *good[i + 1:]) == NULL
        assert fwd(*good[:i], odd, *good[i + 1:]) == INVALID
    for i in (6, 7, 9):
        assert fwd(*good[:i], p + 2, *good[i + 1:]) == INVALID
    good = [plan, ok, ok, ok, ok, ok, None, None, ok, None, ok, ok, ok, ok, ok, None, None]
    for i in (0, 1, 2, 3, 5, 8, 10, 11, 12, 14):
        assert bwd(*good[:i], None, *good[i + 1:]) == NULL
    assert bwd(*good[:4], None, *good[5:]) == NULL  # gradients of g without g
    for i in (1, 4, 8, 10, 13, 14):
        assert bwd(*good[:i], none, *good[i + 1:]) == NULL
        assert bwd(*good[:i], odd, *good[i + 1:]) == INVALID
    for i in (6, 7, 9, 15):
        assert bwd(*good[:i], p + 2, *good[i + 1:]) == INVALID

    def one(q=p, k=p, v=p, g=p, beta=p, state=p, n_slots=4, slots=p, o=p, rows=4, n_h=2, n_hk=1, d_k=8, d_v=8, scale=1.0, dtype=0):
        return step(q, k, v, g, beta, state, n_slots, slots, o, rows, n_h, n_hk, d_k, d_v, scale, dtype, None)
    assert one(rows=0) == 0
    for name in ("q", "k", "v", "beta", "state", "o"):
        assert one(**{name: None}) == NULL
        assert one(**{name: p + 2}) == INVALID
    assert one(rows=-1) == INVALID and one(n_slots=-1) == INVALID and one(n_hk=0) == INVALID and one(n_h=3, n_hk=2) == INVALID
    assert one(slots=None, n_slots=3) == INVALID
    assert one(scale=float("inf")) == INVALID
    assert one(d_k=129) == UNSUPPORTED and one(dtype=7) == UNSUPPORTED and one(rows=1 << 40) == UNSUPPORTED


def test_more_workers_than_travel_with_a_launch():
    """Their table needs a device; without one the call fails cleanly."""
    if torch.cuda.is_available():
        pytest.skip("needs a machine without a GPU")
    P = 20
    many = some(*[0x10000] * P)
    plan = handle(dd.distdl_delta_plan_create(1, 40, 2, 1, 8, 8, P, 1.0, F32))
    assert dd.lib.distdl_delta_fwd(plan, many, many, many, None, many, None, None, many, None, None) in (-6, -7)
    plan = handle(dd.distdl_logits_plan_create(600, 400, P, F32))
    assert dd.lib.distdl_logprob_fwd(plan, many, None, None, 0x20000, None, None, None, 0, 1.0, None) in (-6, -7)
