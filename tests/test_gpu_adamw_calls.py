"""The update's first call on a stream: it makes a table there, and waits for nothing."""
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from test_gpu_adamw import HYPER, make, start8

pytestmark = pytest.mark.gpu
COUNTS = [0, 0, 5, 4096, 0, 4097, 1, 2048, 2049, 0, 100000, 0]


@pytest.mark.parametrize("states8", [False, True])
def test_streams_have_the_same_results(states8):
    """Arrays of no elements among them; each stream's first call and its later ones."""
    require_gpu()
    plan = dd.distdl_adamw_plan_create(COUNTS, torch.float32, states8=states8)
    runs = []
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()):
        d = make(COUNTS, False)
        moments = start8(COUNTS) if states8 else dict(m=d["m"], v=d["v"])
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for step in (1, 2):
                dd.distdl_adamw_step(plan, d["p"], d["g"], **moments, step=step, seed=3, **HYPER)
        torch.cuda.synchronize()
        runs.append([t.view(torch.uint8) for v in [d["p"]] + list(moments.values()) for t in v])
    alone = make(COUNTS, False)
    for i, n in enumerate(COUNTS):  # every array was reached: one by one, with 32-bit moments, gives the same
        if n and not states8:
            one = dd.distdl_adamw_plan_create([n], torch.float32)
            for step in (1, 2):
                dd.distdl_adamw_step(one, [alone["p"][i]], [alone["g"][i]], [alone["m"][i]], [alone["v"][i]], step=step, **HYPER)
            assert torch.equal(alone["p"][i].view(torch.uint8), runs[0][i])
    for run in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], run))


def test_first_call_waits_for_nothing():
    """While the default stream is busy for a fifth of a second, a plan's first call on another stream returns."""
    require_gpu()
    d = make(COUNTS, False)
    warm = dd.distdl_adamw_plan_create(COUNTS, torch.float32)
    stream, a = torch.cuda.Stream(), torch.randn(8192, 8192, device="cuda", dtype=torch.bfloat16)
    b = a @ a
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        dd.distdl_adamw_step(warm, d["p"], d["g"], d["m"], d["v"], step=1, **HYPER)
    torch.cuda.synchronize()
    plan, done = dd.distdl_adamw_plan_create(COUNTS, torch.float32), torch.cuda.Event()
    for _ in range(300):
        torch.matmul(a, a, out=b)
    done.record()
    with torch.cuda.stream(stream):
        dd.distdl_adamw_step(plan, d["p"], d["g"], d["m"], d["v"], step=2, **HYPER)
    waited = done.query()
    torch.cuda.synchronize()
    assert not waited


def test_first_call_cannot_be_recorded():
    require_gpu()
    d = make(COUNTS, False)
    plan, stream, graph, mark = dd.distdl_adamw_plan_create(COUNTS, torch.float32), torch.cuda.Stream(), torch.cuda.CUDAGraph(), torch.zeros(1, device="cuda")
    before = [t.clone() for t in d["p"]]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        mark.add_(1)
        with pytest.raises(dd.DistdlError, match="captured"):
            dd.distdl_adamw_step(plan, d["p"], d["g"], d["m"], d["v"], step=1, **HYPER)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, d["p"]))


@pytest.mark.parametrize("states8", [False, True])
@pytest.mark.parametrize("eps", [1e-30, 1e-42, 1e-60])
def test_weights_without_gradients_under_a_tiny_eps(eps, states8):
    """They only decay, for an eps that 32 bits do not hold either."""
    require_gpu()
    n = 1000
    d = make([n], False)
    d["g"][0][:500], p = 0, d["p"][0].clone()
    moments = start8([n]) if states8 else dict(m=[torch.zeros(n, device="cuda")], v=[torch.zeros(n, device="cuda")])
    plan = dd.distdl_adamw_plan_create([n], torch.float32, states8=states8)
    dd.distdl_adamw_step(plan, d["p"], d["g"], **moments, step=1, **dict(HYPER, eps=eps))
    decay = torch.tensor(1 - HYPER["lr"] * HYPER["weight_decay"], dtype=torch.float64).float().cuda()
    assert torch.equal(d["p"][0][:500], p[:500] * decay) and torch.isfinite(d["p"][0]).all()


def test_copies_of_some_arrays():
    """None among the bf16 copies: that array gets none."""
    require_gpu()
    counts = [300, 5000, 7]
    runs = []
    for some in (False, True):
        d = make(counts, False)
        copies = [torch.full((n,), 7.0, dtype=torch.bfloat16, device="cuda") for n in counts]
        plan = dd.distdl_adamw_plan_create(counts, torch.float32)
        dd.distdl_adamw_step(plan, d["p"], d["g"], d["m"], d["v"], p16=[copies[0], None, copies[2]] if some else copies, step=1, **HYPER)
        runs.append((d["p"], copies))
    (p, full), (p2, partial) = runs
    assert all(torch.equal(a, b) for a, b in zip(p, p2))
    assert torch.equal(full[0], partial[0]) and torch.equal(full[2], partial[2]) and (partial[1] == 7).all() and torch.equal(full[1], p[1].bfloat16())
