"""The gated delta rule with bf16 tensors where results are what is left of numbers that cancel: what stands between the tensors (states, U, P) has 24 bits, as the
header says, so what is left is right however few bits of those numbers it is.

Tolerances.  Every case is the difference of two numbers near 1 + 2^-8, `left` of one to three times 2^-17.  They are exact in three pieces of 8 bits, and so are
products with 1 and -1; four roundings to 24 bits on the way (u = 2^-24 of a number of one) are 4 u / left of the result, 2^-5 at the most, and the result's own rounding
is 2^-8: 2^-4 together.  Of two pieces the second ends with 2^-15, and nothing is left."""
import numpy as np
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TOL = 2.0 ** -4
SIZES = pytest.mark.parametrize("heads, d_k, d_v", [(1, 2, 1), (2, 64, 24), (3, 70, 40), (300, 5, 33)])  # 64 keys and 128, one tile of columns and two


def zeros(heads, d_k, d_v, T=2):
    """Tensors of one sequence of T steps, head by head its keys, to be filled in."""
    return dict(q=torch.zeros(1, T, heads, d_k), k=torch.zeros(1, T, heads, d_k), v=torch.zeros(1, T, heads, d_v), g=torch.zeros(1, T, heads),
                beta=torch.zeros(1, T, heads), h0=torch.zeros(1, heads, d_k, d_v))


def forward(x, scale=1.0):
    n_b, T, heads, d_v = x["v"].shape
    plan = dd.distdl_delta_plan_create(n_b, T, heads, heads, x["q"].shape[3], d_v, 1, scale, BF16)
    on = {n: x[n].cuda().to(BF16 if n in "qkv" else F32) for n in x}
    o = torch.full_like(on["v"], 7.0)
    dd.distdl_delta_fwd(plan, [on["q"]], [on["k"]], [on["v"]], [on["g"]], [on["beta"]], on["h0"], None, [o], None)
    return o.double().cpu().numpy()


def near(got, want):
    want = np.broadcast_to(want, got.shape)
    off = float(np.abs(got / want - 1).max())
    assert off <= TOL


ONE = 1 + 2.0 ** -8
LEFTS = [2.0 ** -17, 2.0 ** -16, 3 * 2.0 ** -17]


@SIZES
def test_outputs_of_states_that_cancel(heads, d_k, d_v):
    """o = scale S^T q with rows 1 + 2^-8 + left and 1 + 2^-8 of S, and q = (1, -1, 0, ...)."""
    require_gpu()
    x = zeros(heads, d_k, d_v)
    lefts = torch.tensor(LEFTS)[torch.arange(d_v) % 3]
    x["h0"][0, :, 0], x["h0"][0, :, 1] = ONE + lefts, ONE
    x["q"][..., 0], x["q"][..., 1] = 1.0, -1.0
    near(forward(x), lefts.double().numpy())


@SIZES
def test_outputs_of_updates_that_cancel(heads, d_k, d_v):
    """Two keys across each other, u_1 = beta_1 = 1 + 2^-8 + left and u_2 = beta_2 = 1 + 2^-8; the second step's o is their difference."""
    require_gpu()
    for left in LEFTS:
        x = zeros(heads, d_k, d_v)
        x["k"][0, 0, :, 0] = x["k"][0, 1, :, 1] = 1.0
        x["beta"][0, 0], x["beta"][0, 1] = ONE + left, ONE
        x["v"][:] = 1.0
        x["q"][0, 1, :, 0], x["q"][0, 1, :, 1] = 1.0, -1.0
        near(forward(x)[0, 1], left)


@SIZES
def test_outputs_of_products_that_cancel(heads, d_k, d_v):
    """The same with u of 1 in both steps and a factor of 1 - left between them, which is in P (a second piece of 1 - left ends with 2^-16)."""
    require_gpu()
    for left in LEFTS:
        x = zeros(heads, d_k, d_v)
        x["k"][0, 0, :, 0] = x["k"][0, 1, :, 1] = 1.0
        x["beta"][:] = 1.0
        x["v"][:] = 1.0
        x["g"][0, 1] = np.log1p(-left)
        x["q"][0, 1, :, 0], x["q"][0, 1, :, 1] = 1.0, -1.0
        near(forward(x)[0, 1], -left)


# ---- gradients: dq and dk of one chunk, in the last column of values; heads that share a key's head add up
GRADIENTS = pytest.mark.parametrize("heads, key_heads, d_k, d_v", [(1, 1, 3, 1), (2, 1, 64, 24), (3, 3, 70, 40), (6, 2, 100, 70), (300, 150, 5, 33)])


def gradients(T, heads, key_heads, d_k, d_v, set_up):
    """(dq, dk) [T, key heads, d_k] over the heads that share them; set_up fills the tensors in."""
    x = zeros(heads, d_k, d_v, T)
    x["q"], x["k"] = (x[n][:, :, :key_heads].clone() for n in "qk")
    x["do"], x["dhT"] = torch.zeros(1, T, heads, d_v), torch.zeros(1, heads, d_k, d_v)
    x["beta"][:] = 1.0
    set_up(x, d_v - 1)
    plan = dd.distdl_delta_plan_create(1, T, heads, key_heads, d_k, d_v, 1, 1.0, BF16)
    on = {n: x[n].cuda().to(BF16 if n in ("q", "k", "v", "do") else F32) for n in x}
    d = {n: [torch.full_like(on[n], 7.0)] for n in ("q", "k", "v", "g", "beta")}
    dd.distdl_delta_bwd(plan, *[[on[n]] for n in ("q", "k", "v", "g", "beta")], on["h0"], None, [on["do"]], on["dhT"], d["q"], d["k"], d["v"], d["g"], d["beta"], None)
    return [d[n][0][0].double().cpu().numpy() / (heads // key_heads) for n in "qk"]


@GRADIENTS
def test_gradients_of_queries_that_cancel(heads, key_heads, d_k, d_v):
    """dq_2 = (do_2 u_1) k_1 + (do_2 u_2) k_2 with k_1 = (1, 1, 0), k_2 = (1, -1, 0), u_1 = 1 + 2^-8 + left and u_2 = -1 - 2^-8."""
    require_gpu()
    for left in LEFTS:
        def set_up(x, col):
            x["k"][0, 0, :, :2], x["k"][0, 1, :, 0], x["k"][0, 1, :, 1] = 1.0, 1.0, -1.0
            x["beta"][0, 0], x["beta"][0, 1] = ONE + left, ONE
            x["v"][0, 0, :, col], x["v"][0, 1, :, col], x["do"][0, 1, :, col] = 1.0, -1.0, 1.0
        near(gradients(2, heads, key_heads, d_k, d_v, set_up)[0][1, :, 0], left)


@GRADIENTS
def test_gradients_of_keys_by_outputs_that_cancel(heads, key_heads, d_k, d_v):
    """dk_1 = (do_1 u_1) q_1 + exp(g_2) (do_2 u_1) q_2 in a place that no key has, with exp(g_2) = 1 - left."""
    require_gpu()
    for left in LEFTS:
        def set_up(x, col):
            x["k"][0, 0, :, 0] = 1.0
            x["q"][0, 0, :, 2], x["q"][0, 1, :, 2] = 1.0, -1.0
            x["g"][0, 1] = np.log1p(-left)
            x["v"][0, 0, :, col] = x["do"][0, 0, :, col] = x["do"][0, 1, :, col] = 1.0
        near(gradients(2, heads, key_heads, d_k, d_v, set_up)[1][0, :, 2], left)


@GRADIENTS
def test_gradients_of_keys_by_earlier_updates_that_cancel(heads, key_heads, d_k, d_v):
    """dk_3 = -(dR_3 u_1) k_1 - (dR_3 u_2) k_2 in a place of k_1 and k_2, with u_1 = 1 + 2^-8 + left, u_2 = -1 - 2^-8, and dR_3 = 1 by the last state's gradient."""
    require_gpu()
    for left in LEFTS:
        def set_up(x, col):
            x["k"][0, 0, :, :2], x["k"][0, 1, :, 0], x["k"][0, 1, :, 1], x["k"][0, 2, :, 2] = 1.0, 1.0, -1.0, 1.0
            x["beta"][0, 0], x["beta"][0, 1] = ONE + left, ONE
            x["v"][0, 0, :, col], x["v"][0, 1, :, col], x["dhT"][0, :, 2, col] = 1.0, -1.0, 1.0
        near(gradients(3, heads, key_heads, d_k, d_v, set_up)[1][2, :, 0], -left)


@GRADIENTS
def test_gradients_of_keys_by_later_updates_that_cancel(heads, key_heads, d_k, d_v):
    """dk_1 = -beta_2 (dR_2 u_1) k_2 - beta_3 (dR_3 u_1) k_3 in a place of k_2 and k_3, with dR_2 = 1, dR_3 = -1, beta_2 = 1 + 2^-8 + left and beta_3 = 1 + 2^-8."""
    require_gpu()
    for left in LEFTS:
        def set_up(x, col):
            x["k"][0, 0, :, 2], x["k"][0, 1, :, :2], x["k"][0, 2, :, 0], x["k"][0, 2, :, 1] = 1.0, 1.0, 1.0, -1.0
            x["beta"][0, 1], x["beta"][0, 2] = ONE + left, ONE
            x["v"][0, 0, :, col], x["dhT"][0, :, 1, col] = 1.0, 1.0
        near(gradients(3, heads, key_heads, d_k, d_v, set_up)[1][0, :, 0], -left)
