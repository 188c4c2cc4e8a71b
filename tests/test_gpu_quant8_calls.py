"""Quantisation of many arrays in one call: recorded without a call before it, over and over, and from several threads."""
import threading

import pytest
import torch

import paper_2006_03108_amd as dd
from gpu_util import require_gpu
from test_gpu_linear8 import empty8

pytestmark = pytest.mark.gpu


def make(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = [torch.randn(3 + i % 7, 5 + 11 * i, generator=g, device="cuda") for i in range(n)]
    x[1 % n] = torch.empty(0, 4, device="cuda")
    if n > 16:
        x[16] = torch.randn(300, 260, generator=g, device="cuda")
    return x


def call(x, outs, tiles=False):
    one, other = outs
    dd.distdl_quant8(x, [t[0] for t in one], [t[1] for t in one], [t[0] for t in other], [t[1] for t in other], tiles=tiles)


def outputs(x, tiles=False):
    return [empty8(*t.shape, tiles) for t in x], [empty8(t.shape[1], t.shape[0], tiles) for t in x]


def same(a, b):
    return all(torch.equal(s, t) for p, q in zip(a, b) for u, v in zip(p, q) for s, t in zip(u, v))


@pytest.mark.parametrize("tiles", [False, True], ids=["rows", "tiles"])
@pytest.mark.parametrize("n", [16, 17, 18, 48, 49, 100])
def test_many_arrays_are_each_alone(n, tiles):
    require_gpu()
    x = make(n, n)
    outs, want = outputs(x, tiles), outputs(x, tiles)
    call(x, outs, tiles)
    for i, t in enumerate(x):
        if t.numel():
            call([t], ([want[0][i]], [want[1][i]]), tiles)
    assert same(outs, want)


def test_recorded_without_an_earlier_call_and_without_end():
    require_gpu()
    stream = torch.cuda.Stream()
    sets = [make(40, s) for s in range(3)]
    outs = [[outputs(x) for _ in range(24)] for x in sets]
    torch.cuda.synchronize()
    graphs = []
    for x, out in zip(sets, outs):
        for o in out:  # 72 recordings of new arrays
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                call(x, o)
            graphs.append(g)
    for _ in range(2):
        for out in outs:
            for o in out:
                for p in o:
                    for q, s in p:
                        q.fill_(0x55), s.fill_(0x55)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for x, out in zip(sets, outs):
            want = outputs(x)
            call(x, want)
            assert all(same(o, want) for o in out)


def test_threads():
    require_gpu()
    sets = [make(40, s) for s in range(4)]
    want = [outputs(x) for x in sets]
    for x, w in zip(sets, want):
        call(x, w)
    torch.cuda.synchronize()
    wrong = []

    def work(x, w):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(30):
                o = outputs(x)
                call(x, o)
                torch.cuda.current_stream().synchronize()
                if not same(o, w):
                    wrong.append(1)

    threads = [threading.Thread(target=work, args=(x, w)) for x, w in zip(sets, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
