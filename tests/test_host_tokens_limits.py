"""The sizes that the header names as the first unsupported ones of the gated delta rule are refused, the last in front of them are not: no device is needed."""
import pytest
import torch

import paper_2006_03108_amd as dd

F32 = torch.float32


def refused(*sizes):
    try:
        dd.distdl_delta_plan_create(*sizes, 1, 1.0, F32)
        return False
    except dd.DistdlError as e:
        assert e.code == -3
        return True


# n_b, T, n_h, n_hk, d_k, d_v
@pytest.mark.parametrize("last, first", [
    ((1, 4, 1, 1, 128, 8), (1, 4, 1, 1, 129, 8)),
    ((1, 4, 1 << 10, 1, 8, 1 << 12), (1, 4, 1 << 10, 1, 8, (1 << 12) + 1)),
    ((1, 4, 1 << 15, 1 << 15, 128, 1), (1, 4, (1 << 15) + 1, (1 << 15) + 1, 128, 1)),
    ((1, 4, 1 << 20, 1, 8, 1), (1, 4, (1 << 20) + 1, 1, 8, 1)),
    ((1, 4, 1, 1, 8, 1 << 20), (1, 4, 1, 1, 8, (1 << 20) + 1)),
    (((1 << 18), 1, 31, 1, 8, 16), ((1 << 18), 1, 32, 1, 8, 16)),
    ((1, 64 * ((1 << 23) - 2), 1, 1, 8, 8), (1, 64 * ((1 << 23) - 1), 1, 1, 8, 8)),
    (((1 << 20) - 1, 1, 1, 1, 8, 8), (1 << 20, 1, 1, 1, 8, 8)),
])
def test_plans_at_the_limits(last, first):
    assert not refused(*last) and refused(*first)


def test_steps_at_the_limits():
    step, p = dd.lib.distdl_delta_step, 0x20000

    def code(rows, n_h, d_k=8, d_v=33):  # (a state that is not aligned is refused behind the sizes: nothing is launched)
        return step(p, p, p, p, p, p + 2, 0, p, p, rows, n_h, 1, d_k, d_v, 1.0, 0, None)
    assert code((1 << 21) - 1, 4) == -1 and code(1 << 21, 4) == -3
    assert code(1, 1, 128) == -1 and code(1, 1, 129) == -3
