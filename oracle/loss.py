"""Token log-probabilities and their gradient, from the definition, in 64 bits."""
import numpy as np


def token_logprob(h, w, target, inv_t=None):
    """h [n, d], w [vocab, d]; returns (logprob, lse) [n], both 0 where target is outside [0, vocab)."""
    h, w, target = np.asarray(h, np.float64), np.asarray(w, np.float64), np.asarray(target)
    n, vocab = len(h), len(w)
    it = np.ones(n) if inv_t is None else np.asarray(inv_t, np.float64)
    lp, lse = np.zeros(n), np.zeros(n)
    for t in range(n):
        if 0 <= target[t] < vocab:
            z = it[t] * (w @ h[t])
            lse[t] = z.max() + np.log(np.exp(z - z.max()).sum())
            lp[t] = z[target[t]] - lse[t]
    return lp, lse


def token_logprob_grad(h, w, target, lse, g, inv_t=None):
    """dL/dh and dL/dw of a loss with dL/dlogprob = g."""
    h, w, target = np.asarray(h, np.float64), np.asarray(w, np.float64), np.asarray(target)
    n, vocab = len(h), len(w)
    it = np.ones(n) if inv_t is None else np.asarray(inv_t, np.float64)
    dh, dw = np.zeros_like(h), np.zeros_like(w)
    for t in range(n):
        if 0 <= target[t] < vocab:
            dz = -np.exp(it[t] * (w @ h[t]) - lse[t])
            dz[target[t]] += 1.0
            dz *= g[t] * it[t]
            dh[t] = dz @ w
            dw += np.outer(dz, h[t])
    return dh, dw
