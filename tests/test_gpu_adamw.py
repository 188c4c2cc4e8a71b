"""AdamW over many arrays on the GPU against the fp64 oracle.

fp32 arithmetic, at most ten roundings between inputs and p: 16 units of 2^-24 of the sizes of its terms.  m and v: 4 units of theirs.
8-bit moments: the new ones are within one code of the unrounded ones, and their mean error over N numbers within four standard
deviations of what rounding at random gives, a code's distance over sqrt(4 N)."""
import numpy as np
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from oracle import blocks

pytestmark = pytest.mark.gpu
UNIT = 2.0 ** -24
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.02)


def host(t):
    return t.float().cpu().double().numpy()


def within(got, want, tol):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, the first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}"


def make(counts, g16, offset=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def new(scale, kind=torch.float32, positive=False):
        ts = []
        for n in counts:
            t = torch.zeros(n + offset, dtype=kind, device="cuda")
            v = scale * torch.randn(n + offset, generator=g, device="cuda")
            t.copy_(v * v if positive else v)
            ts.append(t[offset:])
        return ts

    return dict(p=new(0.1), g=new(0.01, torch.bfloat16 if g16 else torch.float32), m=new(0.01), v=new(0.01, positive=True))


def values8(q, s):
    return blocks.values_of(q.view(torch.uint8).cpu().numpy()[None], s.view(torch.uint8).cpu().numpy()[None], 1, 128)[0]


COUNTS = [1, 7, 128, 129, 4095, 4096, 4097, 0, 20000, 3]


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("g16", [False, True], ids=["g32", "g16"])
def test_32_bit_moments(g16, offset):
    require_gpu()
    d = make(COUNTS, g16, offset)
    before = {k: [host(t) for t in v] for k, v in d.items()}
    copies = [torch.empty(n + offset, dtype=torch.bfloat16, device="cuda")[offset:] for n in COUNTS]
    gscale = torch.full((1,), 0.5, device="cuda")
    plan = dd.distdl_adamw_plan_create(COUNTS, d["g"][0].dtype)
    dd.distdl_adamw_step(plan, d["p"], d["g"], d["m"], d["v"], p16=copies, step=7, gscale=gscale, **HYPER)
    for i in range(len(COUNTS)):
        p, g, m, v = (before[k][i] for k in "pgmv")
        wp, wm, wv = blocks.adamw(p, 0.5 * g, m, v, step=7, **HYPER)
        within(host(d["m"][i]), wm, 4 * UNIT * (np.abs(m) + np.abs(g)))
        within(host(d["v"][i]), wv, 4 * UNIT * (v + g * g))
        within(host(d["p"][i]), wp, 16 * UNIT * (np.abs(p) + np.abs(wp - p) + HYPER["lr"] * 4 * (np.abs(m) + np.abs(g)) / np.sqrt(wv / (1 - 0.99 ** 7))))
        assert torch.equal(copies[i], d["p"][i].bfloat16())


def start8(counts):
    codes = lambda: [torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda") for n in counts]  # noqa: E731
    scales = lambda: [torch.zeros(-(-n // 128), dtype=torch.uint8, device="cuda") for n in counts]  # noqa: E731
    return dict(m=codes(), v=codes(), ms=scales(), vs=scales())


@pytest.mark.parametrize("g16", [False, True], ids=["g32", "g16"])
def test_8_bit_moments(g16):
    require_gpu()
    counts = [n for n in COUNTS if n] + [300000]
    d = make(counts, g16)
    state = start8(counts)
    plan = dd.distdl_adamw_plan_create(counts, d["g"][0].dtype, states8=True)
    for step in (1, 2):
        before = [(host(p), values8(m, ms), values8(v, vs) ** 2) for p, m, ms, v, vs in zip(d["p"], state["m"], state["ms"], state["v"], state["vs"])]
        dd.distdl_adamw_step(plan, d["p"], d["g"], **state, step=step, seed=5, **HYPER)
        for i, (p, m, v) in enumerate(before):
            g = host(d["g"][i])
            wp, wm, wv = blocks.adamw(p, g, m, v, step=step, **HYPER)
            root = np.sqrt(wv)
            within(host(d["p"][i]), wp, 16 * UNIT * (np.abs(p) + np.abs(wp - p)) + 1e-6 * HYPER["lr"] * 40)
            for q, s, want in ((state["m"][i], state["ms"][i], wm), (state["v"][i], state["vs"][i], root)):
                got = values8(q, s)
                unit = (2.0 ** (s.cpu().numpy().astype(float) - 127)).repeat(128)[:got.size]
                code = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(want), 1e-300))) - 3), unit * 2.0 ** -9)
                within(got, want, code * (1 + 1e-5) + 4 * UNIT * np.abs(want))
                if got.size > 10000:
                    z = (got - want) / code
                    assert abs(z.mean()) <= 4 / np.sqrt(4 * z.size) + 2e-3  # (2e-3: 16 of 20 bits of the remainder count; small roots are kept from zero)
                    assert (got[want > 0] > 0).all() if want is root else True


def test_equal_calls_give_equal_bits_and_others_do_not():
    require_gpu()
    counts = [5000, 777]
    runs = []
    for seed, step_on_device in ((1, False), (1, False), (1, True), (2, False)):
        d, state = make(counts, False), start8(counts)
        plan = dd.distdl_adamw_plan_create(counts, torch.float32, states8=True)
        t = torch.zeros(1, dtype=torch.int64, device="cuda")
        for step in (1, 2, 3):
            t += 1
            dd.distdl_adamw_step(plan, d["p"], d["g"], **state, seed=seed, **HYPER, **(dict(step_dev=t) if step_on_device else dict(step=step)))
        runs.append([x.view(torch.uint8) for v in [d["p"]] + list(state.values()) for x in v])
    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))  # noqa: E731
    assert same(runs[0], runs[1]) and same(runs[0], runs[2]) and not same(runs[0], runs[3])


def test_a_moving_average_keeps_its_mean():
    """beta2 = 0.999 moves sqrt(v) by less than a hundredth of a code a step; over 300 steps it has to get where fp32 does."""
    require_gpu()
    n = 1 << 16
    g = torch.Generator(device="cuda").manual_seed(3)
    hyper = dict(HYPER, beta2=0.999, lr=0.0)
    p = [torch.zeros(n, device="cuda")]
    m, v, state = [torch.zeros(n, device="cuda")], [torch.zeros(n, device="cuda")], start8([n])
    plans = [dd.distdl_adamw_plan_create([n], torch.float32, states8=e) for e in (False, True)]
    for step in range(1, 301):
        grad = [torch.randn(n, generator=g, device="cuda") * (1.0 if step <= 100 else 0.1)]
        dd.distdl_adamw_step(plans[0], p, grad, m, v, step=step, **hyper)
        dd.distdl_adamw_step(plans[1], p, grad, **state, step=step, seed=9, **hyper)
    got, want = values8(state["v"][0], state["vs"][0]), np.sqrt(host(v[0]))
    # rounding at random: the mean of the root is kept, its variance (up to a quarter code squared a step, 1/1000 forgotten) adds 5 %
    assert abs(got.mean() / want.mean() - 1) < 0.08


def test_special_values():
    """A NaN gradient stays where it is; an infinite one makes its block's second moment NaN and no other's."""
    require_gpu()
    n = 512
    d, state = make([n], False), start8([n])
    d["g"][0][5], d["g"][0][300] = float("nan"), float("inf")
    plan = dd.distdl_adamw_plan_create([n], torch.float32, states8=True)
    dd.distdl_adamw_step(plan, d["p"], d["g"], **state, step=1, **HYPER)
    bad = torch.zeros(n, dtype=torch.bool)
    bad[5] = bad[300] = True
    assert torch.equal(torch.isnan(d["p"][0]).cpu(), bad)
    m = values8(state["m"][0], state["ms"][0])
    assert np.isnan(m[5]) and np.isfinite(m[:5]).all() and np.isfinite(m[6:256]).all() and np.isnan(m[256:384]).all() and np.isfinite(m[384:]).all()


def test_graph_with_the_step_on_the_device():
    require_gpu()
    counts = [3000, 50]
    runs = []
    for recorded in (False, True):
        d, state, t = make(counts, True), start8(counts), torch.zeros(1, dtype=torch.int64, device="cuda")
        plan = dd.distdl_adamw_plan_create(counts, torch.bfloat16, states8=True)

        def step():
            t.add_(1)
            dd.distdl_adamw_step(plan, d["p"], d["g"], **state, step_dev=t, seed=4, **HYPER)

        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            step()
            if not recorded:
                for _ in range(4):
                    step()
        stream.synchronize()
        if recorded:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                step()
            for _ in range(4):
                graph.replay()
                torch.cuda.synchronize()
        runs.append([x.view(torch.uint8) for v in [d["p"]] + list(state.values()) for x in v])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
