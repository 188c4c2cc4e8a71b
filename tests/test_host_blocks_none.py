"""None among the tensors of a call is NULL, as in the calls of the partitioned layers: no device is needed."""
import torch

import paper_2006_03108_amd as dd
from paper_2006_03108_amd import binding
from test_host_blocks import F32, NULL, code


def test_none_is_null(monkeypatch):
    monkeypatch.setattr(binding, "_stream", lambda: None)  # (asking for the current one needs a device)
    norm = dd.distdl_rmsnorm_plan_create(4, 8, 1, 1e-6, F32)
    assert code(dd.distdl_rmsnorm_fwd, norm, [None], None, [None], None, [None], None, None, None) == NULL
    assert code(dd.distdl_rmsnorm_bwd, norm, [None], [None], None, [None], None, [None], [None]) == NULL
    layer = dd.distdl_linear8_plan_create(4, 8, 8, 1, 1)
    assert code(dd.distdl_linear8_fwd, layer, [None], [None], [None], [None], [None]) == NULL
    assert code(dd.distdl_linear8_bwd_w, layer, [None], [None], [None], [None], [None]) == NULL
    scan = dd.distdl_scan_plan_create(1, 4, 4, 2, "given", F32)
    assert code(dd.distdl_scan_fwd, scan, [None] * 2, [None] * 2, None, None, [None] * 2, None) == NULL
    adam = dd.distdl_adamw_plan_create([4, 4], torch.float32)
    assert code(dd.distdl_adamw_step, adam, *[[None] * 2] * 4, p16=[None, None], lr=1e-3, step=1) == NULL
