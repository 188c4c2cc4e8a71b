"""Steps of the gated delta rule whose beta is 0 or next to it: they add nothing at all, and the gradient of their beta is as right as that of any other, however small
the gradients of the outputs are.  Against the oracle, with the tolerances of test_gpu_delta.py, which are relative: to the norm over these steps alone, and to gradients of the size at hand."""
import numpy as np
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from oracle import tokens
from test_gpu_delta import BF16, F32, limit, make, near, numpy_of, run

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [F32, BF16])


@TYPES
def test_steps_of_beta_zero_add_nothing(dtype):
    """Whatever their values are: 1e35 times a beta of 0 is 0, in the outputs, in the last states and, where nothing else is in them, to the bit."""
    require_gpu()
    x = make(2, 100, 4, 2, 32, 24, dtype, 1, decay=False)
    x["v"][:] = 1e35
    x["beta"][:] = 0.0
    x["h0"][:] = 0.0
    got = run(x, None, 2, 0.3, decay=False, back=False)
    assert (got["o"] == 0).all() and (got["hT"] == 0).all()
    x["h0"] = torch.randn(x["h0"].shape, generator=torch.Generator().manual_seed(2))
    got = run(x, None, 2, 0.3, decay=False, back=False)
    assert torch.equal(got["hT"].cpu(), x["h0"])


@TYPES
@pytest.mark.parametrize("small", [1.0, 1e-9, 1e-12, 1e-18])
@pytest.mark.parametrize("size", [(1, 100, 2, 1, 32, 16, 2), (2, 70, 4, 4, 100, 40, 1), (33, 70, 6, 2, 24, 20, 2)])
def test_gradients_of_a_beta_of_zero(size, small, dtype):
    require_gpu()
    *shape, parts = size
    x = make(*shape, dtype, seed=3)
    T = shape[1]
    kinds = {0: 0.0, 1: 1e-25, 2: -1e-25, 3: 1e-15, 4: -1e-15}  # of eight steps, the others have a beta of size one
    for i, beta in kinds.items():
        x["beta"][:, i::8] = beta
    x["do"], x["dhT"] = (small * x["do"].float()).to(dtype), small * x["dhT"]
    got, n = run(x, None, parts, 0.3), numpy_of(x)
    args = n["q"], n["k"], n["v"], n["g"], n["beta"], n["h0"], np.full(shape[0], T), 0.3
    want = dict(zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), tokens.delta_adjoint(*args, n["do"], n["dhT"])))
    for i in (*kinds, 5):
        near(got["dbeta"][:, i::8] / small, want["dbeta"][:, i::8] / small, limit(got["dbeta"], T), f"dbeta of step {i}", 0.3)
    for name in want:  # (all of them at the size of the gradients)
        near(got[name].float() / small, want[name] / small, limit(got[name], T), name, 0.3 if name in ("dq", "dk", "dv") else 0.0)
