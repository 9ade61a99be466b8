"""Token log-probabilities (GPU) where one token is certain or all but impossible: low temperatures and far logits.

Logits are made of small integers and powers of two, so that every product and sum of them is exact in fp32.  What is left is the arithmetic of the
softmax: a difference z - m is exact; its multiple inv_t log2(e) (z - m) is off by three half steps, 3 2^-24 of it; an exponential by 2^-22 of itself; a
sum of at most 34 values in a lane, then of groups, one by one, 16 and 8 of them, by 64 half steps in all, 2^-18; a logarithm and the last product by 2^-23
of their results."""
import numpy as np
import pytest
import torch

from test_gpu_loss import Call

pytestmark = pytest.mark.gpu
ROWS = [1, 20, 33, 60, 100, 128, 129, 300]            # every form of the forward call
INV_T = [0.7, 1.0, 1.4, 10.0, 1e3, 1e6, 1e9, 1e30]


def exact_batch(n, vocab, d, seed, gap):
    """h, w whose logits are multiples of 2^-6 below 2^8, the largest of a row by about `gap` (0: any); and which entry that is."""
    rng = np.random.default_rng(seed)
    w = rng.integers(-2, 3, size=(vocab, d)) / 16.0
    h = rng.integers(-2, 3, size=(n, d)) / 4.0
    top = rng.integers(0, vocab, n)
    if gap:      # column t is row t's own, with a weight of 4 more for its entry
        assert n <= d
        h[:, :n] = 0
        h[np.arange(n), np.arange(n)] = gap / 4.0
        w[top, np.arange(n)] += 4.0
    return h.astype(np.float32), w.astype(np.float32), top, rng


def reference(h, w, target, it):
    """logprob, lse in 64 bits, and what they may be off by."""
    z = it[:, None].astype(np.float64) * (h.astype(np.float64) @ w.astype(np.float64).T)
    m = z.max(1)
    a = z - m[:, None]
    p = np.exp(a)
    s = p.sum(1)
    lp = a[np.arange(len(h)), target] - np.log(s)
    weighed = (p * -a).sum(1) / s
    off = 3 * 2.0 ** -24 * weighed + 2.0 ** -18 + 2.0 ** -21 * np.log(s)
    return lp, m + np.log(s), off + 2.0 ** -22 * np.abs(lp), off + 2.0 ** -22 * np.abs(m)


@pytest.mark.parametrize("inv_t", INV_T)
@pytest.mark.parametrize("n", ROWS)
def test_log_probabilities_at_low_temperatures(n, inv_t):
    """Any entry as the target: no log-probability is above zero, and each is as exact as its logits."""
    vocab, d = 700, 512
    h, w, top, rng = exact_batch(n, vocab, d, n, 0)
    target = np.where(np.arange(n) % 2, (h @ w.T).argmax(1), top)
    it = np.full(n, inv_t, np.float32)
    c = Call(h, w, target, it)
    c.forward()
    lp, lse = c.results()
    ref_lp, ref_lse, e_lp, e_lse = reference(h, w, target, it)
    assert (lp <= 0).all(), lp.max()
    assert (np.abs(lp - ref_lp) <= e_lp).all(), np.abs(lp - ref_lp).max()
    assert (np.abs(lse - ref_lse) <= e_lse).all(), np.abs(lse - ref_lse).max()


@pytest.mark.parametrize("inv_t", INV_T)
@pytest.mark.parametrize("n", ROWS)
def test_a_certain_token_has_a_log_probability_of_zero(n, inv_t):
    vocab, d = 8192, 512
    h, w, top, rng = exact_batch(n, vocab, d, n, 16)
    z = h.astype(np.float64) @ w.astype(np.float64).T
    others = z.copy()
    others[np.arange(n), top] = -np.inf
    lead = z[np.arange(n), top] - others.max(1)
    assert lead.min() > 5
    it = np.full(n, inv_t, np.float32)
    c = Call(h, w, top, it)
    c.forward()
    lp, lse = c.results()
    ref_lp, ref_lse, e_lp, e_lse = reference(h, w, top, it)
    assert (lp <= 0).all(), lp.max()
    assert (np.abs(lp - ref_lp) <= e_lp).all(), np.abs(lp - ref_lp).max()
    assert (np.abs(lse - ref_lse) <= e_lse).all(), np.abs(lse - ref_lse).max()
    if inv_t >= 10:
        assert (lp == 0).all()      # (the others' exponentials are below 8192 e^-50)


@pytest.mark.parametrize("n", [20, 60, 128, 300])
def test_the_largest_inverse_temperatures(n):
    """Up to the largest number of fp32: the logits' multiples overflow, their differences' exponentials are zero or one."""
    vocab, d = 700, 512
    h, w, top, rng = exact_batch(n, vocab, d, n, 16)
    it = np.full(n, 3.0e38, np.float32)
    it[::2] = np.finfo(np.float32).max
    target = np.where(np.arange(n) % 3 == 0, (top + 1) % vocab, top)
    c = Call(h, w, target, it)
    c.forward()
    lp, lse = c.results()
    assert (lp[target == top] == 0).all() and (lp[target != top] == -np.inf).all()
    assert (lse == np.inf).all()
    c.backward(c.lse[:n].clone(), torch.ones(n, device="cuda"))
    assert np.isnan(c.gradients()[0]).all()      # (an infinite lse says nothing of the probabilities)


def gradients(h, w, target, it, g, lse):
    """G, dh, dw in 64 bits; lse in 64 bits too."""
    z = it[:, None].astype(np.float64) * (h.astype(np.float64) @ w.astype(np.float64).T)
    G = -np.exp(z - lse[:, None])
    G[np.arange(len(h)), target] += 1
    G *= (g.astype(np.float64) * it)[:, None]
    return G, G @ w.astype(np.float64), G.T @ h.astype(np.float64)


@pytest.mark.parametrize("inv_t", [10.0, 1e3, 1e6, 1e9, 1e30])
@pytest.mark.parametrize("n", ROWS)
def test_gradients_where_one_token_is_certain(n, inv_t):
    """A certain token's gradient vanishes, that of an impossible target is g inv_t (w[target] - w[certain]): whatever lse, a number of 32 bits, is off by."""
    vocab, d = 700, 512
    h, w, top, rng = exact_batch(n, vocab, d, n, 16)
    target = np.where(rng.random(n) < 0.5, top, (top + 1 + rng.integers(0, vocab - 1, n)) % vocab)
    it = np.full(n, inv_t, np.float32)
    g = rng.normal(size=n).astype(np.float32)
    c = Call(h, w, target, it)
    c.forward()
    c.backward(c.lse[:n].clone(), torch.from_numpy(g).cuda())
    dh, dw = c.gradients()
    _, true_lse, _, _ = reference(h, w, target, it)
    G, ref_h, ref_w = gradients(h, w, target, it, g, true_lse)
    # entries of G are g inv_t, minus it, or below 1e-40 of it; g inv_t is rounded (2^-24) and, to bf16, once more; sums and results as anywhere
    G = np.where(np.abs(G) < 1e-30 * np.abs(g * it.astype(np.float64))[:, None], 0, G)
    e_G = (2.0 ** -8 + 2.0 ** -23) * np.abs(G)
    for got, ref, e in ((dh, G @ w, e_G @ np.abs(w) + (vocab + 64) * 2.0 ** -24 * (np.abs(G) @ np.abs(w))),
                        (dw, G.T @ h, e_G.T @ np.abs(h) + (n + 64) * 2.0 ** -24 * (np.abs(G).T @ np.abs(h)))):
        assert (np.abs(got - ref) <= e + 2.0 ** -8 * (np.abs(ref) + e) + 1e-38 * inv_t).all(), np.abs(got - ref).max() / inv_t
    assert (np.abs(dh[target == top]) <= 1e-30 * inv_t).all()


@pytest.mark.parametrize("n", [20, 100, 300])
def test_gradients_of_far_logits(n):
    """Logits of thousands at a temperature of one, and a row whose logits are all equal."""
    vocab, d = 700, 512
    h, w, top, rng = exact_batch(n, vocab, d, n, 16)
    h *= 512
    h[0] = 0
    target = np.where(np.arange(n) % 2, top, (top + 7) % vocab)
    it = np.ones(n, np.float32)
    g = rng.normal(size=n).astype(np.float32)
    c = Call(h, w, target, None)
    c.forward()
    lp, lse = c.results()
    ref_lp, true_lse, e_lp, e_lse = reference(h, w, target, it)
    assert (lp <= 0).all() and (np.abs(lp - ref_lp) <= e_lp).all() and (np.abs(lse - true_lse) <= e_lse).all()
    c.backward(c.lse[:n].clone(), torch.from_numpy(g).cuda())
    dh, dw = c.gradients()
    G, ref_h, ref_w = gradients(h, w, target, it, g, true_lse)
    # (of the row of equal logits: e^-lse is off by what lse, 6.6, is rounded by, and an exponential's 2^-20)
    e_G = (2.0 ** -8 + 2.0 ** -19) * np.abs(G) + 2.0 ** -22 * np.abs(g)[:, None] * (np.abs(G) > 0)
    for got, ref, e in ((dh, ref_h, e_G @ np.abs(w) + (vocab + 64) * 2.0 ** -24 * (np.abs(G) @ np.abs(w))),
                        (dw, ref_w, e_G.T @ np.abs(h) + (n + 64) * 2.0 ** -24 * (np.abs(G).T @ np.abs(h)))):
        assert (np.abs(got - ref) <= e + 2.0 ** -8 * (np.abs(ref) + e) + 1e-30).all(), np.abs(got - ref).max()
    certain = (target == top) & (np.arange(n) > 0)
    assert certain.any() and (np.abs(dh[certain]) <= 1e-30).all()
