"""Pins of the oracle of the operators of a model of tokens: closed forms, brute force, and differences."""
import numpy as np

from oracle import tokens


def test_a_delta_step_replaces_what_a_key_holds():
    """With a factor of 1, beta of 1 and a key of length 1 the state answers the key with the value, and keys across it as before."""
    rng = np.random.default_rng(0)
    S, k, v = rng.normal(size=(1, 6, 4)), rng.normal(size=6), rng.normal(size=(1, 4))
    k = (k / np.linalg.norm(k))[None]
    o, after = tokens.delta_step(S, k, k, v, np.ones(1), np.ones(1), 1.0)
    assert np.allclose(o, v)
    other = rng.normal(size=6)
    other -= (other @ k[0]) * k[0]
    assert np.allclose(after[0].T @ other, S[0].T @ other)


def test_delta_without_updates_decays():
    g = np.full((1, 5, 2), -0.3)
    h0 = np.random.default_rng(1).normal(size=(1, 2, 3, 4))
    q = np.ones((1, 5, 1, 3))
    o, hT = tokens.delta_forward(q, q, np.ones((1, 5, 2, 4)), g, np.zeros((1, 5, 2)), h0, np.array([4]), 1.0)
    assert np.allclose(hT, h0 * np.exp(-1.2))
    assert np.allclose(o[0, 2], np.exp(-0.9) * h0[0].sum(1)) and (o[0, 4] == 0).all()


def test_delta_is_linear_attention_for_orthogonal_keys():
    """Keys of unit length across each other find nothing to replace: o_t = scale sum over j <= t of beta_j (q_t k_j) v_j."""
    rng = np.random.default_rng(2)
    T, d = 6, 8
    k = np.linalg.qr(rng.normal(size=(d, d)))[0][:T]
    q, v, beta = rng.normal(size=(T, d)), rng.normal(size=(T, 3)), rng.random(T)
    o, _ = tokens.delta_forward(q[None, :, None], k[None, :, None], v[None, :, None], np.zeros((1, T, 1)), beta[None, :, None], np.zeros((1, 1, d, 3)), np.array([T]), 0.5)
    want = 0.5 * (np.tril(q @ k.T) * beta) @ v
    assert np.allclose(o[0, :, 0], want)


def test_delta_adjoint_of_shared_keys_and_lengths():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(2, 4, 1, 3)), 0.5 * rng.normal(size=(2, 4, 1, 3)), rng.normal(size=(2, 4, 2, 2))
    ins = [q, k, v, -rng.random((2, 4, 2)), rng.random((2, 4, 2)), rng.normal(size=(2, 2, 3, 2))]
    do, dhT, ends = rng.normal(size=v.shape), rng.normal(size=ins[5].shape), np.array([4, 2])
    value = lambda a: sum((x * w).sum() for x, w in zip(tokens.delta_forward(*a, ends, 0.6), (do, dhT)))  # noqa: E731
    grads = tokens.delta_adjoint(*ins, ends, 0.6, do, dhT)
    for i, g in enumerate(grads):
        direction = rng.normal(size=g.shape)
        at = lambda s: value([x + s * direction if j == i else x for j, x in enumerate(ins)])  # noqa: E731
        assert abs((at(1e-5) - at(-1e-5)) / 2e-5 - (g * direction).sum()) < 1e-7
    assert all((g[1, 2:] == 0).all() for g in grads[:5])


def test_log_probabilities():
    x = np.log(np.array([[0.5, 0.25, 0.125, 0.125], [1.0, 1.0, 0.0, 2.0]]) + 0.0 + np.array([[0], [0]]), where=np.array([[1, 1, 1, 1], [1, 1, 0, 1]], bool),
               out=np.full((2, 4), -np.inf))
    logp, lse, entropy, order, top = tokens.logprob_forward(x, np.array([1, -1]), 4)
    assert np.allclose(logp, [np.log(0.25), 0.0]) and np.allclose(lse, [0.0, np.log(4.0)])
    assert np.allclose(entropy, [np.log(2) * 1.75, np.log(2) * 1.5])
    assert order.tolist() == [[0, 1, 2, 3], [3, 0, 1, 2]]
    assert np.allclose(top[1, :3], np.log([0.5, 0.25, 0.25])) and np.isneginf(top[1, 3])


def test_a_row_of_nothing():
    x = np.full((1, 3), -np.inf)
    logp, lse, entropy, order, top = tokens.logprob_forward(x, np.array([1]), 2)
    assert np.isneginf(logp[0]) and np.isneginf(lse[0]) and entropy[0] == 0 and order.tolist() == [[0, 1]] and np.isneginf(top).all()
    assert (tokens.logprob_adjoint(x, np.array([1]), np.ones(1), np.ones(1)) == 0).all()


def test_divergence_of_a_distribution_from_itself_and_from_another():
    rng = np.random.default_rng(4)
    x = rng.normal(size=(2, 5))
    ids = np.tile(np.arange(5), (2, 1))
    loss, dx = tokens.distill(x, ids, x + 3.0, np.ones(2), 1.3)
    assert np.allclose(loss, 0) and np.allclose(dx, 0)
    t = rng.normal(size=(2, 3))
    ids = np.array([[0, 3, 3], [4, -1, 9]])
    value = lambda x: (tokens.distill(x, ids, t, np.ones(2), 0.7)[0] * [0.5, 2.0]).sum()  # noqa: E731
    _, dx = tokens.distill(x, ids, t, np.array([0.5, 2.0]), 0.7)
    for i in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[i] = 1e-6
        assert abs((value(x + d) - value(x - d)) / 2e-6 - dx[i]) < 1e-7
    loss, _ = tokens.distill(x, ids, t, np.ones(2))
    assert np.isclose(loss[1], -tokens.log_softmax(x)[0][1, 4])  # one place: the cross entropy
