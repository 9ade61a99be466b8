"""Entries of the vocabulary that are masked by an infinite weight on a channel that is 1 for every position: their logits are -infinity, their
probabilities 0 (GPU, against the softmax over the other entries in 64 bits)."""
import numpy as np
import pytest
import torch

from test_gpu_loss import Call
from test_gpu_loss_low_temperature import exact_batch, gradients, reference

pytestmark = pytest.mark.gpu

# (a thread of the join takes every 128th group of 64: group 128 behind group 0, 129 behind 1)
VOCAB, D = 9000, 256
MASKS = {"first group": slice(0, 64), "second group": slice(64, 128), "group 128": slice(8192, 8256), "two groups and more": slice(100, 300), "last entries": slice(8930, 9000),
         "a whole tile": slice(8448, 8704), "first and last": slice(0, 9000, 8999), "all but one": slice(1, 9000), "every second": slice(0, 9000, 2)}


def masked_batch(n, mask, seed):
    h, w, _, rng = exact_batch(n, VOCAB, D, seed, 0)
    h[:, 5] = 1.0
    w[:, 5] = 0.0
    out = np.zeros(VOCAB, bool)
    out[mask] = True
    target = np.flatnonzero(~out)[rng.integers(0, (~out).sum(), n)]
    blocked = w.copy()
    blocked[out, 5] = -np.inf
    it = (1 / (0.7 + 0.3 * rng.random(n))).astype(np.float32)
    return h, w, blocked, out, target, it, rng


def renumbered(out, target):
    """A target's number among the entries that are left."""
    return (np.cumsum(~out) - 1)[target]


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("n", [1, 20, 60, 128, 300])
def test_masked_entries_leave_the_others_their_log_probabilities(n, mask):
    h, w, blocked, out, target, it, rng = masked_batch(n, MASKS[mask], n)
    c = Call(h, blocked, target, it)
    c.forward()
    lp, lse = c.results()
    ref_lp, ref_lse, e_lp, e_lse = reference(h, w[~out], renumbered(out, target), it)
    assert (np.abs(lp - ref_lp) <= e_lp).all() and (np.abs(lse - ref_lse) <= e_lse).all()


@pytest.mark.parametrize("n", [20, 60, 300])
def test_a_masked_target_is_impossible_and_all_masked_entries_are_no_distribution(n):
    h, w, blocked, out, target, it, rng = masked_batch(n, slice(64, 192), 7 + n)
    target[::3] = 100
    c = Call(h, blocked, target, it)
    c.forward()
    lp, lse = c.results()
    assert (lp[::3] == -np.inf).all() and np.isfinite(lse).all() and np.isfinite(lp[1::3]).all()
    blocked[:, 5] = -np.inf
    c = Call(h, blocked, target, it)
    c.forward()
    lp, lse = c.results()
    assert (lse == -np.inf).all() and np.isnan(lp).all()


@pytest.mark.parametrize("n", [20, 60, 300])
@pytest.mark.parametrize("entry", [70, 8300])
def test_a_nan_beside_masked_entries_is_not_lost(n, entry):
    """One entry whose weight is NaN, in a group that is masked but for it: no position has a sum."""
    h, w, blocked, out, target, it, rng = masked_batch(n, slice(64, 8700), 9 + n)
    blocked[entry, 5] = np.nan
    c = Call(h, blocked, target, it)
    c.forward()
    lp, lse = c.results()
    assert np.isnan(lp).all() and np.isnan(lse).all()


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("n", [1, 20, 60, 128, 200, 300])
def test_masked_entries_have_no_gradient(n, mask):
    """dw of masked entries is 0 and that of the others as without them, whatever rows the call is padded to.  (dh is G w: 0 times infinity.)"""
    h, w, blocked, out, target, it, rng = masked_batch(n, MASKS[mask], 20 + n)
    g = rng.normal(size=n).astype(np.float32)
    c = Call(h, blocked, target, it)
    c.forward()
    c.backward(c.lse[:n].clone(), torch.from_numpy(g).cuda(), dh=False)
    dw = c.gradients()[1]
    _, ref_lse, _, _ = reference(h, w[~out], renumbered(out, target), it)
    G, _, ref = gradients(h, w[~out], renumbered(out, target), it, g, ref_lse)
    scale = np.abs(g * it)[:, None]
    e_G = 2.0 ** -8 * np.abs(G) + 2.0 ** -18 * scale
    e = e_G.T @ np.abs(h) + (n + 64) * 2.0 ** -24 * (np.abs(G).T @ np.abs(h))
    assert (dw[out] == 0).all()
    assert (np.abs(dw[~out] - ref) <= e + 2.0 ** -8 * (np.abs(ref) + e)).all()


@pytest.mark.parametrize("mask", ["first group", "group 128", "last entries", "all but one", "every second"])
@pytest.mark.parametrize("n", [1, 20, 60, 128, 300])
def test_masks_of_the_lowest_number(n, mask):
    """The lowest bf16 number as the weight: logits that an inverse temperature above 1 takes beyond fp32.  Here dh, with 0 times that number, is of the others."""
    h, w, blocked, out, target, it, rng = masked_batch(n, MASKS[mask], 40 + n)
    blocked[out, 5] = float(torch.finfo(torch.bfloat16).min)
    g = rng.normal(size=n).astype(np.float32)
    c = Call(h, blocked, target, it)
    c.forward()
    lp, lse = c.results()
    left = renumbered(out, target)
    ref_lp, ref_lse, e_lp, e_lse = reference(h, w[~out], left, it)
    assert (np.abs(lp - ref_lp) <= e_lp).all() and (np.abs(lse - ref_lse) <= e_lse).all()
    c.backward(c.lse[:n].clone(), torch.from_numpy(g).cuda())
    dh, dw = c.gradients()
    G, ref_h, ref_w = gradients(h, w[~out], left, it, g, ref_lse)
    e_G = 2.0 ** -8 * np.abs(G) + 2.0 ** -18 * np.abs(g * it)[:, None]
    e_h = e_G @ np.abs(w[~out]) + (VOCAB + 64) * 2.0 ** -24 * (np.abs(G) @ np.abs(w[~out]))
    e_w = e_G.T @ np.abs(h) + (n + 64) * 2.0 ** -24 * (np.abs(G).T @ np.abs(h))
    assert (dw[out] == 0).all()
    assert (np.abs(dw[~out] - ref_w) <= e_w + 2.0 ** -8 * (np.abs(ref_w) + e_w)).all()
    assert (np.abs(dh - ref_h) <= e_h + 2.0 ** -8 * (np.abs(ref_h) + e_h)).all()


@pytest.mark.parametrize("n", [1, 20, 60, 128, 300])
def test_masks_at_an_inverse_temperature_of_zero(n):
    """All entries but those masked by an infinity are equally likely, those of the lowest number among them; nothing has a gradient."""
    h, w, blocked, out, target, it, rng = masked_batch(n, slice(8192, 8400), 60 + n)
    it[:] = 0.0
    target[1::3] = 8200
    for weight, left in ((-np.inf, VOCAB - 208), (float(torch.finfo(torch.bfloat16).min), VOCAB)):
        blocked[out, 5] = weight
        c = Call(h, blocked, target, it)
        c.forward()
        lp, lse = c.results()
        of_masked = (target == 8200) & (weight == -np.inf)
        # (a sum of ones, exact; a logarithm's 2^-22, and the lowest number's 5e-7)
        assert (np.abs(lse - np.log(left)) <= 2.0 ** -22 * np.log(left) + 1e-6).all()
        assert (np.abs(lp[~of_masked] + np.log(left)) <= 2.0 ** -22 * np.log(left) + 1e-6).all() and (lp[of_masked] == -np.inf).all()
        c.backward(c.lse[:n].clone(), torch.ones(n, device="cuda"), dh=weight != -np.inf)
        dh, dw = c.gradients()
        assert (dw == 0).all() and (weight == -np.inf or (dh == 0).all())
