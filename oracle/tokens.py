"""Operators of a recurrent model that answers with tokens, in fp64 numpy, from their formulas: the gated delta rule, log probabilities
with entropy and alternatives, and the divergence from a teacher's top logits.  Whole tensors; what is split over workers is cut by the caller."""
import numpy as np


# ---- gated delta rule -----------------------------------------------------

def delta_step(state, q, k, v, a, beta, scale):
    """(o, state after) of one step; state [..., d_k, d_v], q and k [..., d_k], v [..., d_v], a and beta [...]."""
    before = a[..., None, None] * state
    u = beta[..., None] * (v - np.einsum("...kv,...k->...v", before, k))
    after = before + k[..., :, None] * u[..., None, :]
    return scale * np.einsum("...kv,...k->...v", after, q), after


def _per_head(x, n_h):
    return x.repeat(n_h // x.shape[2], 2)


def delta_forward(q, k, v, g, beta, h0, lengths, scale):
    """(o, last states); q, k [n, steps, key heads, d_k], v [n, steps, heads, d_v], g (log of the factors) and beta [n, steps, heads]."""
    n_h = v.shape[2]
    q, k = _per_head(q, n_h), _per_head(k, n_h)
    o, state = np.zeros_like(v), h0.copy()
    for t in range(v.shape[1]):
        live = lengths > t
        o[live, t], state[live] = delta_step(state[live], q[live, t], k[live, t], v[live, t], np.exp(g[live, t]), beta[live, t], scale)
    return o, state


def delta_adjoint(q, k, v, g, beta, h0, lengths, scale, do, dhT):
    """Gradients of q, k, v, g, beta and h0 for gradients do of all outputs and dhT of the last states."""
    n, T, n_h, _ = v.shape
    n_hk = q.shape[2]
    q, k, a = _per_head(q, n_h), _per_head(k, n_h), np.exp(g)
    states = [h0.copy()]
    for t in range(T):
        live, after = lengths > t, states[-1].copy()
        after[live] = delta_step(after[live], q[live, t], k[live, t], v[live, t], a[live, t], beta[live, t], scale)[1]
        states.append(after)
    dq, dk, dv, dg, dbeta, dS = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros_like(g), np.zeros_like(beta), dhT.copy()
    for t in range(T - 1, -1, -1):
        for i in np.nonzero(lengths > t)[0]:
            for h in range(n_h):
                before, kt, b = a[i, t, h] * states[t][i, h], k[i, t, h], beta[i, t, h]
                r = v[i, t, h] - before.T @ kt
                dq[i, t, h] = scale * (states[t + 1][i, h] @ do[i, t, h])
                D = dS[i, h] + scale * np.outer(q[i, t, h], do[i, t, h])
                du = D.T @ kt
                dk[i, t, h] = D @ (b * r) - before @ (b * du)
                dv[i, t, h], dbeta[i, t, h] = b * du, du @ r
                D = D - np.outer(kt, b * du)
                dg[i, t, h] = (D * before).sum()
                dS[i, h] = a[i, t, h] * D
    shared = lambda x: x.reshape(n, T, n_hk, n_h // n_hk, -1).sum(3)  # noqa: E731
    return shared(dq), shared(dk), dv, dg, dbeta, dS


# ---- log probabilities ----------------------------------------------------

def log_softmax(x, temperature=1.0):
    """(log p, lse); a row of -inf alone has -inf in both."""
    z = x / temperature
    most = z.max(1, keepdims=True)
    most = np.where(np.isneginf(most), 0.0, most)
    with np.errstate(divide="ignore"):
        total = np.log(np.exp(z - most).sum(1, keepdims=True))
    with np.errstate(invalid="ignore"):  # (a maximum of -1e20 plus a logarithm is -1e20, so log p is not z - lse)
        return np.where(np.isneginf(total), -np.inf, (z - most) - total), (most + total)[:, 0]


def _plogp(log_p):
    with np.errstate(invalid="ignore"):
        return np.where(np.isneginf(log_p), 0.0, np.exp(log_p) * log_p)


def logprob_forward(x, targets, n_top, temperature=1.0):
    """(log p of the targets, lse, entropy, places of the n_top largest, their log p); equal values in the order of their places."""
    log_p, lse = log_softmax(x, temperature)
    live = (targets >= 0) & (targets < x.shape[1])
    logp = np.where(live, log_p[np.arange(len(x)), np.where(live, targets, 0)], 0.0)
    order = np.argsort(-x, axis=1, kind="stable")[:, :n_top]
    return logp, lse, -_plogp(log_p).sum(1), order, np.take_along_axis(log_p, order, 1)


def logprob_adjoint(x, targets, dlogp, dentropy, temperature=1.0):
    log_p, lse = log_softmax(x, temperature)
    p, plogp = np.exp(log_p), _plogp(log_p)
    live = (targets >= 0) & (targets < x.shape[1])
    weight = np.where(live, dlogp, 0.0)[:, None]
    dz = -weight * p - dentropy[:, None] * (plogp - p * plogp.sum(1, keepdims=True))
    dz[np.nonzero(live)[0], targets[live]] += weight[live, 0]
    return np.where(np.isneginf(lse)[:, None], 0.0, dz / temperature)


# ---- distillation ---------------------------------------------------------

def distill(x, ids, teacher, weight, temperature=1.0):
    """(loss of each row, gradient of weight * loss)."""
    log_p, lse = log_softmax(x, temperature)
    loss, dx = np.zeros(len(x)), np.zeros_like(x)
    for r in range(len(x)):
        used = (ids[r] >= 0) & (ids[r] < x.shape[1])
        t = np.where(used, teacher[r] / temperature, -np.inf)
        if np.isneginf(t.max()):
            continue
        t = np.exp(t - t.max())
        t /= t.sum()
        for k in np.nonzero(t)[0]:
            loss[r] += t[k] * (np.log(t[k]) - log_p[r, ids[r, k]])
        if weight[r] != 0 and not np.isneginf(lse[r]):
            dx[r] = np.exp(log_p[r])
            np.add.at(dx[r], ids[r][used], -t[used])
            dx[r] *= weight[r] / temperature
    return loss, dx
