"""Entries of the vocabulary that are masked by an infinite weight on a channel that is 1 for every position: their logits are -infinity, their
probabilities 0 (GPU, against the softmax over the other entries in 64 bits)."""
import numpy as np
import pytest
import torch

from test_gpu_loss import Call
from test_gpu_loss_low_temperature import exact_batch, reference

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
