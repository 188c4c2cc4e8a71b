"""Arrays of more than 2^32 bytes: what the operators give at their far end is what a call on that end alone gives.

The same kernels sum in the same order there, so results have to be equal bit for bit, but where a comment says otherwise."""
import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def rnd(*s, dtype=torch.bfloat16, seed=0):
    t = torch.empty(*s, dtype=dtype, device="cuda")
    return t.normal_(generator=torch.Generator(device="cuda").manual_seed(seed))


def test_norm():
    require_gpu()
    rows, n_f, end = 700_000, 4096, 96
    x, r = rnd(rows, n_f), rnd(rows, n_f, seed=1)
    g = 1 + 0.1 * rnd(n_f, dtype=torch.float32, seed=2)

    def run(x, r):
        plan = dd.distdl_rmsnorm_plan_create(len(x), n_f, 1, 1e-5, torch.bfloat16)
        s, y, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        q, qs = torch.empty(x.shape, dtype=torch.uint8, device="cuda"), torch.empty(n_f // 128, len(x), dtype=torch.uint8, device="cuda")
        rstd = torch.empty(len(x), device="cuda")
        dd.distdl_rmsnorm_fwd(plan, [x], [r], [g], [s], [y], [q], [qs], rstd)
        dd.distdl_rmsnorm_bwd(plan, [s], [g], rstd, [y], [r], [dx], [torch.empty_like(g)])
        return [s[-end:], y[-end:], q[-end:], qs[:, -end:], rstd[-end:], dx[-end:]]

    want = run(x[-end:].clone(), r[-end:].clone())
    assert all(torch.equal(a, b) for a, b in zip(run(x, r), want))


@pytest.mark.parametrize("tiles", [False, True], ids=["rows", "tiles"])
def test_quantisation(tiles):
    require_gpu()
    rows, cols, end = 2336 * 128, 8192, 128
    x = rnd(rows, cols)

    def run(x):
        n = len(x)
        byte = lambda *s: torch.empty(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
        q, qt = byte(n, cols), byte(cols, n)
        s, st = (byte(n // 128, cols // 128), byte(cols // 128, n // 128)) if tiles else (byte(cols // 128, n), byte(n // 128, cols))
        dd.distdl_quant8([x], [q], [s], [qt], [st], tiles=tiles)
        return [q[-end:], qt[:, -end:], s[-1:] if tiles else s[:, -end:], st[:, -1:] if tiles else st[-1:]]

    want = run(x[-end:].clone())
    assert all(torch.equal(a, b) for a, b in zip(run(x), want))


def test_product():
    """Tiles of other sizes sum in another order: each of the K / 32 steps is off by a unit of 2^-23 of the sum of magnitudes at most."""
    require_gpu()
    rows, K, N, end = 1_100_000, 4096, 128, 256
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randint(0, 64, (rows, K), generator=g, device="cuda", dtype=torch.uint8)
    w = torch.randint(0, 64, (N, K), generator=g, device="cuda", dtype=torch.uint8)
    xs = torch.randint(124, 130, (K // 128, rows), generator=g, device="cuda", dtype=torch.uint8)
    ws = torch.randint(124, 130, (1, K // 128), generator=g, device="cuda", dtype=torch.uint8)

    def run(x, xs):
        plan = dd.distdl_linear8_plan_create(len(x), K, N, 1, 1, torch.float32)
        y = torch.empty(len(x), N, device="cuda")
        dd.distdl_linear8_fwd(plan, [x], [xs], [w], [ws], [y])
        return y[-end:]

    want = run(x[-end:].clone(), xs[:, -end:].contiguous())
    got = run(x, xs)  # (codes below 64 are positive: the sum is that of magnitudes)
    assert ((got - want).abs() <= 2 * K // 32 * 2.0 ** -23 * want).all()


def scan(n, T, C, a, x, dh, end):
    plan = dd.distdl_scan_plan_create(n, T, C, 1, "sigmoid", torch.bfloat16)
    h, da, dx = [[torch.empty_like(x)] for _ in range(3)]
    dd.distdl_scan_fwd(plan, [a], [x], None, None, h, None)
    dd.distdl_scan_bwd(plan, [a], [x], h, None, None, [dh], None, da, dx, None)
    return [end(t[0]) for t in (h, da, dx)]


def test_scan_of_many_chains():
    require_gpu()
    n, T, C, k = 600, 2000, 2048, 10
    a, x, dh = [rnd(n, T, C, seed=s) for s in range(3)]
    want = scan(k, T, C, *[t[-k:].clone() for t in (a, x, dh)], lambda t: t)
    assert all(torch.equal(u, v) for u, v in zip(scan(n, T, C, a, x, dh, lambda t: t[-k:].clone()), want))


def test_scan_of_few_chains():
    """A call on the last steps alone starts from zero, which gates of 1 / (1 + exp(-g)), g ~ N(0, 1), have forgotten after 1000 steps; its runs of
    tiles begin elsewhere, so the state in 32 bits differs in its last places and a bf16 result by one rounding (2^-7 and 1e-5 of the size 1
    of a state).  The adjoint starts at the end in both: where it reads the same states it is equal."""
    require_gpu()
    T, C, end = 150016, 16384, 4096
    a, x, dh = [rnd(1, T, C, seed=s) for s in range(3)]
    late = lambda t: t[:, -end // 2:].clone()  # noqa: E731
    h, da, dx = scan(1, T, C, a, x, dh, late)
    wh, wa, wx = scan(1, end, C, *[t[:, -end:].clone() for t in (a, x, dh)], late)
    assert ((h.float() - wh.float()).abs() <= 2.0 ** -7 * wh.float().abs() + 1e-5).all()
    assert torch.equal(dx, wx)
    same = torch.cat([torch.zeros_like(h[:, :1], dtype=torch.bool), h[:, :-1] == wh[:, :-1]], 1)
    assert torch.equal(da[same], wa[same])


@pytest.mark.parametrize("states8", [False, True], ids=["32", "8"])
def test_update(states8):
    """With 8-bit moments the rounding is a function of a number's place; the weights are made before it."""
    require_gpu()
    count, end = (4_400_000_000, 1 << 20) if states8 else (1_200_000_000, 1 << 20)
    p = rnd(count, dtype=torch.float32)
    g = rnd(count, seed=1) if states8 else rnd(count, dtype=torch.float32, seed=1)

    def run(p, g):
        n = p.numel()
        plan = dd.distdl_adamw_plan_create([n], g.dtype, states8)
        kind = torch.uint8 if states8 else torch.float32
        m, v = torch.zeros(n, dtype=kind, device="cuda"), torch.zeros(n, dtype=kind, device="cuda")
        ms, vs = [[torch.zeros(-(-n // 128), dtype=torch.uint8, device="cuda")] for _ in range(2)] if states8 else (None, None)
        dd.distdl_adamw_step(plan, [p], [g], [m], [v], ms, vs, None, lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=1)
        return [p[-end:]] + ([] if states8 else [m[-end:], v[-end:]])

    want = run(p[-end:].clone(), g[-end:].clone())
    assert all(torch.equal(u, w) for u, w in zip(run(p, g), want))
