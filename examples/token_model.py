"""A model of tokens on virtual workers: time on two of them, the vocabulary on three.  A student learns from a teacher's top logits, then answers token by token.

    x = embedding[token];  n = RMS norm of x;  q, k, v, gates = W n;  q, k: RMS norm of each head, to unit length
    o = gated delta rule over q, k, v with g = -softplus(gate), beta = sigmoid(gate);  y = x + W_o o;  logits = W_v (RMS norm of y)

The teacher's logits go through distdl_logprob_fwd, which leaves the best tokens and their log probabilities; the student's loss and gradient against
them are one call of distdl_distill_fwd_bwd.  Every time worker has its own rows; weight gradients are sum-reduced over them.

    python examples/token_model.py [--steps 100]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2006_03108_amd as dd  # noqa: E402

EPS = 1e-6
F32 = torch.float32


def split(n, parts):
    return [n // parts + (r < n % parts) for r in range(parts)]


class Model:
    """n_b sequences of T tokens; heads of d_k keys and d_v values.  Weights are a dict of fp32 tensors."""

    def __init__(self, n_b, T, vocab=301, d=48, heads=4, key_heads=2, d_k=16, d_v=24, workers=2, vocab_workers=3, seed=0):
        assert T % workers == 0, "every time worker has the same steps here"
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.n_b, self.T, self.vocab, self.d, self.P, self.V = n_b, T, vocab, d, workers, vocab_workers
        self.heads, self.key_heads, self.d_k, self.d_v = heads, key_heads, d_k, d_v
        self.parts = split(vocab, vocab_workers)
        new = lambda *s: torch.randn(*s, generator=g, device="cuda") / s[-1] ** 0.5  # noqa: E731
        self.weights = {"embedding": torch.randn(vocab, d, generator=g, device="cuda"), "q": new(key_heads * d_k, d), "k": new(key_heads * d_k, d),
                        "v": new(heads * d_v, d), "gates": new(2 * heads, d), "out": new(d, heads * d_v),
                        **{f"head{i}": 2 * new(n, d) for i, n in enumerate(self.parts)}, "norm1": torch.ones(d, device="cuda"), "norm2": torch.ones(d, device="cuda")}
        self.unit = torch.full((d_k,), d_k ** -0.5, device="cuda")  # an RMS norm times this has length 1
        self.plans = {}
        self.scan = dd.distdl_delta_plan_create(n_b, T, heads, key_heads, d_k, d_v, workers, d_k ** -0.5, F32)
        counts = [w.numel() for w in self.weights.values()]
        self.adam = dd.distdl_adamw_plan_create(counts, F32)
        self.m, self.v_ = ([torch.zeros(n, device="cuda") for n in counts] for _ in range(2))
        self.step_number = 0

    def plan(self, kind, rows):
        """Plans by the rows of a call, made once."""
        if (kind, rows) not in self.plans:
            d, h, hk, dk, dv = self.d, self.heads, self.key_heads, self.d_k, self.d_v
            affine = {"q": (d, hk * dk, 1), "k": (d, hk * dk, 1), "v": (d, h * dv, 1), "gates": (d, 2 * h, 1), "out": (h * dv, d, 1), "head": (d, self.vocab, self.V)}
            if kind in affine:
                n_fi, n_fo, parts = affine[kind]
                self.plans[kind, rows] = dd.distdl_affine_plan_create(rows, n_fi, n_fo, parts, 1, F32)
            elif kind == "logits":
                self.plans[kind, rows] = dd.distdl_logits_plan_create(rows, self.vocab, self.V, F32)
            else:
                self.plans[kind, rows] = dd.distdl_rmsnorm_plan_create(rows * (hk if kind == "heads" else 1), dk if kind == "heads" else d, 1, EPS, F32)
        return self.plans[kind, rows]

    # ---- pieces of a pass, for the rows of one worker ----

    def affine(self, name, x, W):
        rows = x.shape[0]
        y = [torch.empty(rows, w.shape[0], device="cuda") for w in W]
        dd.distdl_affine_fwd(self.plan(name, rows), [x], W, None, y)
        return y

    def affine_back(self, name, x, W, dy):
        dx, dW = torch.empty_like(x), [torch.empty_like(w) for w in W]
        dd.distdl_affine_bwd(self.plan(name, x.shape[0]), [x], W, dy, [dx], dW, None)
        return dx, dW

    def norm(self, kind, rows, x, gain):
        y, rstd = torch.empty_like(x), torch.empty(x.numel() // gain.numel(), device="cuda")
        dd.distdl_rmsnorm_fwd(self.plan(kind, rows), [x], None, [gain], None, [y], None, None, rstd)
        return y, rstd

    def norm_back(self, kind, rows, x, gain, rstd, dy, dsum=None):
        dx, dg = torch.empty_like(x), torch.empty_like(gain)
        dd.distdl_rmsnorm_bwd(self.plan(kind, rows), [x], [gain], rstd, [dy], None if dsum is None else [dsum], [dx], [dg])
        return dx, dg

    def before(self, tokens):
        """What the recurrence needs of a worker's tokens, [rows]."""
        w, rows = self.weights, tokens.numel()
        s = {"tokens": tokens, "x": w["embedding"][tokens]}
        s["n"], s["rstd"] = self.norm("rows", rows, s["x"], w["norm1"])
        for name in ("q", "k", "v", "gates"):
            s[name + "0"] = self.affine(name, s["n"], [w[name]])[0]
        for name in ("q", "k"):
            s[name], s["rstd_" + name] = self.norm("heads", rows, s[name + "0"], self.unit)
        a, b = s["gates0"].chunk(2, 1)
        s["g"], s["beta"] = -torch.nn.functional.softplus(a).contiguous(), torch.sigmoid(b).contiguous()
        return s

    def after(self, s, o):
        """Logits of a worker's rows, the vocabulary on its workers."""
        w, rows = self.weights, s["x"].shape[0]
        s["o"] = o
        s["y"] = s["x"] + self.affine("out", o, [w["out"]])[0]
        s["n2"], s["rstd2"] = self.norm("rows", rows, s["y"], w["norm2"])
        return self.affine("head", s["n2"], [w[f"head{i}"] for i in range(self.V)])

    def forward(self, tokens):
        """tokens: [n_b, T].  (what the adjoint needs, logits of every time worker)"""
        states = [self.before(t.reshape(-1)) for t in tokens.chunk(self.P, 1)]
        arrays = {n: [s[n] for s in states] for n in ("q", "k", "g", "beta")} | {"v": [s["v0"] for s in states]}
        o = [torch.empty_like(v) for v in arrays["v"]]
        self.last = torch.empty(self.n_b, self.heads, self.d_k, self.d_v, device="cuda")
        dd.distdl_delta_fwd(self.scan, arrays["q"], arrays["k"], arrays["v"], arrays["g"], arrays["beta"], None, None, o, self.last)
        return states, [self.after(s, t) for s, t in zip(states, o)]

    def backward(self, states, dlogits):
        """Gradients of all weights, each time worker's part sum-reduced over the workers."""
        w, parts, d_o = self.weights, [], []
        for s, dx in zip(states, dlogits):
            rows, g = s["x"].shape[0], {}
            head = [w[f"head{i}"] for i in range(self.V)]
            dn, dW = self.affine_back("head", s["n2"], head, dx)
            g.update({f"head{i}": t for i, t in enumerate(dW)})
            s["dy"], g["norm2"] = self.norm_back("rows", rows, s["y"], w["norm2"], s["rstd2"], dn)
            do, (g["out"],) = self.affine_back("out", s["o"], [w["out"]], [s["dy"]])
            d_o.append(do)
            parts.append(g)
        of = lambda n: [s[n] for s in states]  # noqa: E731
        like = lambda n: [torch.empty_like(s[n]) for s in states]  # noqa: E731
        dq, dk, dv, dg, db = (like(n) for n in ("q", "k", "v0", "g", "beta"))
        dd.distdl_delta_bwd(self.scan, of("q"), of("k"), of("v0"), of("g"), of("beta"), None, None, d_o, None, dq, dk, dv, dg, db, None)
        for i, (s, g) in enumerate(zip(states, parts)):
            rows = s["x"].shape[0]
            a, _ = s["gates0"].chunk(2, 1)
            back = {"v": dv[i], "gates": torch.cat([-dg[i] * torch.sigmoid(a), db[i] * s["beta"] * (1 - s["beta"])], 1)}
            for name, d in (("q", dq[i]), ("k", dk[i])):
                back[name], _ = self.norm_back("heads", rows, s[name + "0"], self.unit, s["rstd_" + name], d)
            dn = torch.zeros_like(s["n"])
            for name, d in back.items():
                part, (g[name],) = self.affine_back(name, s["n"], [w[name]], [d])
                dn += part
            dx, g["norm1"] = self.norm_back("rows", rows, s["x"], w["norm1"], s["rstd"], dn, s["dy"])
            g["embedding"] = torch.zeros_like(w["embedding"]).index_put_((s["tokens"],), dx, accumulate=True)
        grads = {n: torch.empty_like(t) for n, t in w.items()}
        dd.distdl_sumreduce_fwd([p[n] for n in grads for p in parts], list(grads.values()), self.P)
        return grads

    def best(self, tokens, n_top):
        """A teacher's answer: places and log probabilities of its best tokens, for every time worker."""
        out = []
        for x in self.forward(tokens)[1]:
            rows = x[0].shape[0]
            ids, logp = torch.empty(rows, n_top, dtype=torch.int32, device="cuda"), torch.empty(rows, n_top, device="cuda")
            dd.distdl_logprob_fwd(self.plan("logits", rows), x, None, None, None, None, ids, logp)
            out.append((ids, logp))
        return out

    def distil(self, tokens, best, temperature=1.0):
        """(mean loss, gradients) against a teacher's best tokens."""
        states, logits = self.forward(tokens)
        losses, weight = [], torch.full((tokens.numel() // self.P,), 1 / tokens.numel(), device="cuda")
        for x, (ids, logp) in zip(logits, best):
            losses.append(torch.empty_like(weight))
            dd.distdl_distill_fwd_bwd(self.plan("logits", weight.numel()), x, ids, logp, weight, losses[-1], x, temperature)  # (the gradient takes the logits' place)
        return torch.cat(losses).mean(), self.backward(states, logits)

    def likelihood(self, tokens, targets, entropy_weight=0.0):
        """(mean of -log p(target) - entropy_weight entropy, gradients); a target of -1 counts for nothing."""
        states, logits = self.forward(tokens)
        total, n = 0.0, tokens.numel()
        for x, t in zip(logits, targets.chunk(self.P, 1)):
            t = t.reshape(-1).to(torch.int32)
            plan, (logp, lse, entropy) = self.plan("logits", t.numel()), (torch.empty(t.numel(), device="cuda") for _ in range(3))
            dd.distdl_logprob_fwd(plan, x, t, logp, lse, entropy)
            total = total - (logp.sum() + entropy_weight * entropy.sum()) / n
            dd.distdl_logprob_bwd(plan, x, t, lse, entropy, torch.full_like(logp, -1 / n), torch.full_like(logp, -entropy_weight / n), x)
        return total, self.backward(states, logits)

    def update(self, grads, lr):
        self.step_number += 1
        flat = lambda ts: [t.view(-1) for t in ts]  # noqa: E731
        dd.distdl_adamw_step(self.adam, flat(self.weights.values()), flat(grads.values()), self.m, self.v_, lr=lr, step=self.step_number)

    def decode(self, tokens, pool, slots):
        """Logits of one token for each row; the states of the sequences lie in pool at slots."""
        s = self.before(tokens)
        rows, shape = tokens.numel(), (tokens.numel(), self.heads, self.d_v)
        o = torch.empty(shape, device="cuda")
        dd.distdl_delta_step(s["q"].view(rows, self.key_heads, self.d_k), s["k"].view(rows, self.key_heads, self.d_k), s["v0"].view(shape), s["g"], s["beta"], pool,
                             slots, o, self.d_k ** -0.5)
        return self.after(s, o.view(rows, -1))


def run(steps=100, n_b=4, T=96, say=None):
    """(losses, largest difference of decoding from the chunked pass, largest logit)"""
    teacher, student = Model(n_b, T, seed=1), Model(n_b, T, seed=2)
    losses = []
    for i in range(steps):
        tokens = torch.randint(0, student.vocab, (n_b, T), generator=torch.Generator(device="cuda").manual_seed(i), device="cuda")
        loss, grads = student.distil(tokens, teacher.best(tokens, 16))
        student.update(grads, 3e-3)
        losses.append(float(loss))
        if say and i % 20 == 0:
            say(f"step {i}: loss {losses[-1]:.4f}")
    logits = torch.cat([torch.cat([t.view(n_b, T // student.P, -1) for t in x], 2) for x in student.forward(tokens)[1]], 1)
    pool, slots = torch.zeros(n_b + 3, student.heads, student.d_k, student.d_v, device="cuda"), torch.arange(n_b, dtype=torch.int32, device="cuda") + 2
    off = max(float((torch.cat(student.decode(tokens[:, t], pool, slots), 1) - logits[:, t]).abs().max()) for t in range(T))
    return losses, off, float(logits.abs().max())


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=100)
    losses, off, size = run(ap.parse_args().steps, say=lambda m: print(m, flush=True))
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}; decoding differs from the chunked pass by {off:.2g} of {size:.2g}")
