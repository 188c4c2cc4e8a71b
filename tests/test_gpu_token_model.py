"""The operators together: a model of tokens on workers, its gradients and its decoding."""
import os
import sys

import numpy as np
import pytest
import torch

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_the_example_runs_and_decodes():
    """Decoding computes the same sums in another order: 96 steps of numbers of size one, and logits as sums of 48 of them, each rounded by 2^-24 of
    its size at most a hundred times in a row: 1e-4 of the largest."""
    require_gpu()
    import token_model
    losses, off, size = token_model.run(steps=3, T=96)
    assert all(np.isfinite(losses))
    assert off <= 1e-4 * size


def case():
    import token_model
    model, teacher = token_model.Model(2, 70, seed=3), token_model.Model(2, 70, seed=4)
    g = torch.Generator(device="cuda").manual_seed(5)
    tokens = torch.randint(0, model.vocab, (2, 70), generator=g, device="cuda")
    return model, tokens, torch.randint(-1, model.vocab, (2, 70), generator=g, device="cuda"), teacher.best(tokens, 9)


def calls(model, tokens, targets, best, what):
    return (lambda: model.distil(tokens, best, 1.5)) if what == "distil" else (lambda: model.likelihood(tokens, targets, 0.1))


def plain_loss(model, w, tokens, targets, best, what):
    """The model's formulas, step by step, in fp64 on the host."""
    n_b, T, hk, h, d_k, d_v = *tokens.shape, model.key_heads, model.heads, model.d_k, model.d_v
    norm = lambda x: x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    x = w["embedding"][tokens]
    n = norm(x) * w["norm1"]
    q, k = (norm((n @ w[i].t()).view(n_b, T, hk, d_k)).repeat_interleave(h // hk, 2) * d_k ** -0.5 for i in "qk")
    v = (n @ w["v"].t()).view(n_b, T, h, d_v)
    a, b = (n @ w["gates"].t()).chunk(2, 2)
    decay, beta = torch.exp(-torch.nn.functional.softplus(a)), torch.sigmoid(b)
    S, o = x.new_zeros(n_b, h, d_k, d_v), []
    for t in range(T):
        S = S * decay[:, t, :, None, None]
        u = beta[:, t, :, None] * (v[:, t] - (k[:, t, :, :, None] * S).sum(2))
        S = S + k[:, t, :, :, None] * u[:, :, None]
        o.append(d_k ** -0.5 * (q[:, t, :, :, None] * S).sum(2))
    y = x + torch.stack(o, 1).reshape(n_b, T, -1) @ w["out"].t()
    z = norm(y) * w["norm2"] @ torch.cat([w[f"head{i}"] for i in range(model.V)]).t()
    if what == "likelihood":
        logp = z.log_softmax(-1)
        return -(logp.gather(2, targets.clamp(min=0)[..., None])[..., 0] * (targets >= 0) - 0.1 * (logp.exp() * logp).sum(-1)).mean()
    join = lambda i: torch.cat([p[i].view(n_b, T // model.P, -1) for p in best], 1).cpu()  # noqa: E731
    t = (join(1).double() / 1.5).log_softmax(-1)
    return (t.exp() * (t - (z / 1.5).log_softmax(-1).gather(2, join(0).long()))).sum(-1).mean()


@pytest.mark.parametrize("what", ["distil", "likelihood"])
def test_gradients_are_those_of_the_formulas(what):
    """Ten operators in a row, each right to 2e-5 of its own size at most (their own tests' bound for fp32) and to a tenth of that as a rule: 1e-4."""
    require_gpu()
    model, tokens, targets, best = case()
    loss, grads = calls(model, tokens, targets, best, what)()
    w = {n: t.double().cpu().requires_grad_() for n, t in model.weights.items()}
    want = plain_loss(model, w, tokens.cpu(), targets.cpu(), best, what)
    want.backward()
    assert abs(float(loss) - want.item()) <= 1e-5 * max(1, abs(want.item()))
    for n, t in w.items():
        assert float((grads[n].double().cpu() - t.grad).norm()) <= 1e-4 * float(t.grad.norm()), n


@pytest.mark.parametrize("what", ["distil", "likelihood"])
def test_gradients_are_differences(what):
    """Along the gradient of each tensor, by 2e-3 of a length of one both ways: the loss is known to 1e-6 (a mean of sums in fp32), so the quotient over 4e-3
    to 5e-4, and (2e-3)^2 / 6 of a third derivative of a hundred adds less than 1e-4."""
    require_gpu()
    model, tokens, targets, best = case()
    f = calls(model, tokens, targets, best, what)
    _, grads = f()
    way = {n: t / t.norm() for n, t in grads.items()}
    slope = sum(float(t.double().norm()) for t in grads.values())

    def at(step):
        kept = {n: w.clone() for n, w in model.weights.items()}
        for n, w in model.weights.items():
            w += step * way[n]
        value = float(f()[0])
        for n, w in model.weights.items():
            w.copy_(kept[n])
        return value
    got = (at(2e-3) - at(-2e-3)) / 4e-3
    assert abs(got - slope) <= 1e-3 * slope + 6e-4, (got, slope)


def test_a_teacher_that_is_the_student_asks_for_nothing_but_what_it_did_not_store():
    """With all tokens stored, the divergence of a model from itself is 0, and so is its gradient."""
    require_gpu()
    import token_model
    model = token_model.Model(2, 16, vocab=60, seed=6)
    tokens = torch.randint(0, 60, (2, 16), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    loss, grads = model.distil(tokens, model.best(tokens, 60))
    assert abs(float(loss)) <= 1e-5
    assert all(float(t.abs().max()) <= 1e-6 for t in grads.values())
