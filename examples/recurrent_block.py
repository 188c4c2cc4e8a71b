"""A gated recurrent block, trained and decoded on virtual workers that share time.

    s = RMS norm of x;   [a, u] = W1 s   (8-bit operands; worker 0 of the outputs holds gates, worker 1 inputs)
    h_t = sigmoid(a_t) h_{t-1} + (1 - sigmoid(a_t)) u_t      (time on P workers, the state passes from one to the next)
    y = W2 h                                                 (8-bit operands)

Every time worker has its own rows; weight gradients are sum-reduced over the workers, and one AdamW call with 8-bit moments updates all
weights.  The task: leaky averages of the input with a decay for each channel, which is what the block can express.  After
training, tokens are decoded one at a time from a pool of states.

    python examples/recurrent_block.py [--steps 300]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2006_03108_amd as dd  # noqa: E402

EPS = 1e-6


def blocks(n):
    return -(-n // dd.BLOCK8)


def codes(rows, cols, tiles=False):
    """Codes and scales of a matrix, in blocks of its rows or in tiles."""
    return (torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device="cuda"),
            torch.empty((blocks(rows), blocks(cols)) if tiles else (blocks(cols), rows), dtype=torch.uint8, device="cuda"))


class Block:
    def __init__(self, n_b, T, d, workers=2, seed=0):
        assert T % workers == 0, "every time worker has the same steps here"
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
        self.n_b, self.T, self.d, self.P, self.rows = n_b, T, d, workers, n_b * T // workers
        w1 = [torch.randn(d, d, generator=g, device="cuda") / d ** 0.5 for _ in range(2)]
        w2 = torch.randn(d, d, generator=g, device="cuda") / d ** 0.5
        self.weights = [*w1, w2, torch.ones(d, device="cuda")]  # gates, inputs, outputs, gains
        self.norm = dd.distdl_rmsnorm_plan_create(self.rows, d, 1, EPS, torch.float32)
        self.mix = dd.distdl_linear8_plan_create(self.rows, d, 2 * d, 2, 1, torch.float32)
        self.out = dd.distdl_linear8_plan_create(self.rows, d, d, 1, 1, torch.float32)
        self.scan = dd.distdl_scan_plan_create(n_b, T, d, workers, "sigmoid", torch.float32)
        counts = [w.numel() for w in self.weights]
        self.adam = dd.distdl_adamw_plan_create(counts, torch.float32, states8=True)
        state = lambda: [torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda") for n in counts]  # noqa: E731
        scale = lambda: [torch.zeros(blocks(n), dtype=torch.uint8, device="cuda") for n in counts]  # noqa: E731
        self.moments = dict(m=state(), v=state(), ms=scale(), vs=scale())
        self.q = [(codes(d, d, True), codes(d, d, True)) for _ in range(3)]  # each product's weights, and their transposes
        R, each = self.rows, range(workers)
        self.sq, self.hq = [codes(R, d) for _ in each], [codes(R, d) for _ in each]
        self.st, self.ht = [codes(d, R) for _ in each], [codes(d, R) for _ in each]
        self.dq, self.dt = [[codes(R, d) for _ in range(3)] for _ in each], [[codes(d, R) for _ in range(3)] for _ in each]
        act = lambda: [new(n_b, T // workers, d) for _ in each]  # noqa: E731
        self.s, self.a, self.u, self.h, self.y, self.dy, self.dh, self.da, self.du, self.ds, self.dx = (act() for _ in range(11))
        self.rstd, self.last = [new(R) for _ in each], new(n_b, d)
        self.parts = [[torch.empty_like(w) for w in self.weights] for _ in each]  # each time worker's gradients
        self.grads = [torch.empty_like(w) for w in self.weights]
        self.loss = torch.zeros(1, dtype=torch.float64, device="cuda")
        self.step_number = 0
        self.quantise()

    def quantise(self):
        one, other = [q[0] for q in self.q], [q[1] for q in self.q]
        dd.distdl_quant8(self.weights[:3], [t[0] for t in one], [t[1] for t in one], [t[0] for t in other], [t[1] for t in other], tiles=True)

    def matrix(self, t):
        return t.view(-1, self.d)

    def forward(self, x):
        for p in range(self.P):
            s = self.matrix(self.s[p])
            dd.distdl_rmsnorm_fwd(self.norm, [self.matrix(x[p])], None, [self.weights[3]], None, [s], [self.sq[p][0]], [self.sq[p][1]], self.rstd[p])
            dd.distdl_linear8_fwd(self.mix, [self.sq[p][0]], [self.sq[p][1]], [self.q[0][0][0], self.q[1][0][0]], [self.q[0][0][1], self.q[1][0][1]],
                                  [self.matrix(self.a[p]), self.matrix(self.u[p])])
        dd.distdl_scan_fwd(self.scan, self.a, self.u, None, None, self.h, self.last)
        for p in range(self.P):
            dd.distdl_quant8([self.matrix(self.h[p])], [self.hq[p][0]], [self.hq[p][1]], [self.ht[p][0]], [self.ht[p][1]])
            dd.distdl_linear8_fwd(self.out, [self.hq[p][0]], [self.hq[p][1]], [self.q[2][0][0]], [self.q[2][0][1]], [self.matrix(self.y[p])])
        return self.y

    def train(self, x, target, lr):
        """One step on the mean squared error; the loss stays on the device."""
        self.forward(x)
        dd.distdl_mse_fwd_bwd(self.y, target, self.dy, self.loss)
        for p in range(self.P):
            (q, qt), (gate, into, out, _) = (self.dq[p], self.dt[p]), self.parts[p]
            dd.distdl_quant8([self.matrix(self.dy[p])], [q[2][0]], [q[2][1]], [qt[2][0]], [qt[2][1]])
            dd.distdl_linear8_bwd_x(self.out, [q[2][0]], [q[2][1]], [self.q[2][1][0]], [self.q[2][1][1]], [self.matrix(self.dh[p])])
            dd.distdl_linear8_bwd_w(self.out, [qt[2][0]], [qt[2][1]], [self.ht[p][0]], [self.ht[p][1]], [out])
        dd.distdl_scan_bwd(self.scan, self.a, self.u, self.h, None, None, self.dh, None, self.da, self.du, None)
        for p in range(self.P):
            (q, qt), (gate, into, _, gain) = (self.dq[p], self.dt[p]), self.parts[p]
            dd.distdl_quant8([self.matrix(self.da[p]), self.matrix(self.du[p])], [q[0][0], q[1][0]], [q[0][1], q[1][1]],
                             [qt[0][0], qt[1][0]], [qt[0][1], qt[1][1]])
            dd.distdl_quant8([self.matrix(self.s[p])], None, None, [self.st[p][0]], [self.st[p][1]])
            dd.distdl_linear8_bwd_x(self.mix, [q[0][0], q[1][0]], [q[0][1], q[1][1]], [self.q[0][1][0], self.q[1][1][0]],
                                    [self.q[0][1][1], self.q[1][1][1]], [self.matrix(self.ds[p])])
            dd.distdl_linear8_bwd_w(self.mix, [qt[0][0], qt[1][0]], [qt[0][1], qt[1][1]], [self.st[p][0]], [self.st[p][1]], [gate, into])
            dd.distdl_rmsnorm_bwd(self.norm, [self.matrix(x[p])], [self.weights[3]], self.rstd[p], [self.matrix(self.ds[p])], None,
                                  [self.matrix(self.dx[p])], [gain])
        # the sum-reduce of the weights' gradients over the time workers
        dd.distdl_sumreduce_fwd([self.parts[p][i] for i in range(4) for p in range(self.P)], self.grads, self.P)
        self.step_number += 1
        dd.distdl_adamw_step(self.adam, self.weights, self.grads, **self.moments, lr=lr, beta2=0.99, step=self.step_number, seed=7)
        self.quantise()
        return self.loss

    def decode(self, x, pool, slots):
        """Outputs of one token for each row of x [rows, d]; the states of the sequences lie in pool at slots."""
        rows, d = x.shape
        norm = dd.distdl_rmsnorm_plan_create(rows, d, 1, EPS, torch.float32)
        mix, out = (dd.distdl_linear8_plan_create(rows, d, n * d, n, 1, torch.float32) for n in (2, 1))
        q, (a, u, h, y) = codes(rows, d), (torch.empty_like(x) for _ in range(4))
        dd.distdl_rmsnorm_fwd(norm, [x], None, [self.weights[3]], None, None, [q[0]], [q[1]], None)
        dd.distdl_linear8_fwd(mix, [q[0]], [q[1]], [self.q[0][0][0], self.q[1][0][0]], [self.q[0][0][1], self.q[1][0][1]], [a, u])
        dd.distdl_scan_step(a, u, pool, slots, h, "sigmoid")
        dd.distdl_quant8([h], [q[0]], [q[1]], None, None)
        dd.distdl_linear8_fwd(out, [q[0]], [q[1]], [self.q[2][0][0]], [self.q[2][0][1]], [y])
        return y


def batch(n_b, T, d, workers, seed):
    """Inputs and their leaky averages, cut over the time workers."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n_b, T, d, generator=g, device="cuda")
    keep, state, target = torch.linspace(0.5, 0.95, d, device="cuda"), torch.zeros(n_b, d, device="cuda"), torch.empty_like(x)
    for t in range(T):
        state = keep * state + (1 - keep) * x[:, t]
        target[:, t] = state
    cut = lambda v: [t.contiguous() for t in v.chunk(workers, 1)]  # noqa: E731
    return cut(x), cut(target)


def run(steps=300, n_b=8, T=64, d=128, workers=2, say=None):
    """(first loss, last loss, largest difference of decoding from the scan)"""
    block, losses = Block(n_b, T, d, workers), []
    for i in range(steps):
        x, target = batch(n_b, T, d, workers, i)
        losses.append(float(block.train(x, target, lr=1e-2 * (1 - i / steps))))
        if say and i % 50 == 0:
            say(f"step {i}: loss {losses[-1]:.5f}")
    x, target = batch(n_b, T, d, workers, steps)
    y = torch.cat(block.forward(x), 1)
    whole, pool, slots = torch.cat(x, 1), torch.zeros(n_b + 4, d, device="cuda"), torch.arange(n_b, dtype=torch.int32, device="cuda") + 2
    off = max(float((block.decode(whole[:, t].contiguous(), pool, slots) - y[:, t]).abs().max()) for t in range(T))
    return losses[0], losses[-1], off, float(y.abs().max())


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=300)
    first, last, off, size = run(ap.parse_args().steps, say=lambda m: print(m, flush=True))
    print(f"loss {first:.5f} -> {last:.5f}; decoding differs from the scan by {off:.2g} of {size:.2g}")
