"""Windowed attention and attention over shared prompts where scores are so large that a maximum in powers of two, rounded to 32 bits, is far from what it rounds."""
import numpy as np
import pytest
import torch

import paper_2509_19128_amd as pl

from paged_util import bf16, i32, pool_of

pytestmark = pytest.mark.gpu

PEAK = {32: 23296.0, 64: 19456.0, 128: 16256.0}   # bf16 numbers whose products' sum, scaled and rounded, is off by 2^7 and more (worked out with whole numbers)


def _attend(q, k, v, hd):
    """q [Hq], k [positions, Hkv]: what all elements of a head are, but for their signs, which q and k have in common.  Their products have 16 bits and the sums of up
    to 128 of them 23, so scores are exact in 32 bits.  The result in 64 bits and its error, that of the exponents being: scale and differences 2^-22 of an exponent that
    still counts (150 at most), and the roundings of two maxima below 2^10, where weights are relative to such: 2^-12 covers both."""
    Hkv = k.shape[1]
    s = q.reshape(Hkv, -1)[:, :, None] * k.T[:, None] * hd      # [Hkv, G, positions], whole in 64 bits
    w = np.exp((s - s.max(-1, keepdims=True)) / np.sqrt(hd))
    w /= w.sum(-1, keepdims=True)
    out = np.einsum("hgt,thd->hgd", w, v)
    e = np.einsum("hgt,thd->hgd", w * (2.0 ** -8 + 2 * 2.0 ** -12 + (len(k) + 64) * 2.0 ** -24), np.abs(v))
    # weights below 2^-126 are none in 32 bits, beside a sum of 1 at least
    e += 2.0 ** -126 * np.abs(v).sum(0)[:, None]
    return out.reshape(-1, hd), (e + 2.0 ** -8 * (np.abs(out) + e)).reshape(-1, hd)


class Batch:
    """Rows of `lens` positions, of which the first `prompt` are the same; keys by levels[b] (position -> what every element of the key is)."""

    def __init__(self, q, levels, hd, page, prompt=0, seed=0):
        rng = np.random.default_rng(seed)
        self.n, self.Hq = q.shape
        self.hd, self.page, self.prompt, self.q = hd, page, prompt, q.astype(np.float64)
        self.k = [np.asarray(a, np.float64) for a in levels]
        self.lens = [len(a) for a in self.k]
        Hkv = self.Hkv = self.k[0].shape[1]
        sign = rng.choice([-1.0, 1.0], hd)
        self.v = [rng.integers(-8, 9, (c, Hkv, hd)).astype(np.float64) for c in self.lens]
        for a in (self.k, self.v):
            for x in a:
                x[:prompt] = a[0][:prompt]
        self.pages = (512 << 20) // (self.n * Hkv * hd * 4 * page) + 1 + -(-max(self.lens) // page)   # (a call that shares)
        self.most = self.pages * page
        used = [-(-c // page) for c in self.lens]
        whole = prompt // page
        table, at = np.full((self.n, self.pages), -1), whole
        for b, u in enumerate(used):
            table[b, :whole] = np.arange(whole)
            table[b, whole:u] = np.arange(at, at + u - whole)
            at += u - whole
        K = [k[:, :, None] * sign for k in self.k]
        self.pool = pool_of(K, self.v, [t[:u] for t, u in zip(table, used)], at, page)
        _, self.qd = bf16(q[:, :, None] * sign)
        assert np.array_equal(self.qd[:, :, 0].float().cpu().numpy() * sign[0], q)   # (nothing was rounded)
        self.td, self.cd = i32(table), i32(self.lens)

    def _ws(self, size):
        return torch.full((size,), 0xA5, device="cuda", dtype=torch.uint8)

    def _cache(self):
        return self.qd.data_ptr(), self.pool.data_ptr(), self.td.data_ptr(), self.cd.data_ptr()

    def check(self, out, window=None, sinks=0):
        torch.cuda.synchronize()
        got = out.float().cpu().numpy()
        for b in range(self.n):
            j = np.arange(self.lens[b])
            see = j if window is None else j[(j < sinks) | (j >= self.lens[b] - window)]
            ref, e = _attend(self.q[b], self.k[b][see], self.v[b][see], self.hd)
            bad = np.argwhere(~(np.abs(got[b] - ref) <= e))
            assert len(bad) == 0, (b, len(bad), *[(*at, x[tuple(at)]) for at in bad[:1] for x in (got[b], ref, e)])

    def window(self, window, sinks, most=None):
        most = most or max(self.lens)
        shape = (self.n, self.Hq, self.Hkv, self.hd)
        ws = self._ws(pl.pl_attention_window_workspace_bytes(*shape, most, window, sinks))
        out = torch.zeros(self.n, self.Hq, self.hd, device="cuda", dtype=torch.bfloat16)
        pl.pl_attention_window(*self._cache(), out.data_ptr(), ws.data_ptr(), *shape, self.page, self.pages, most, window, sinks)
        self.check(out, window, sinks)

    def shared(self):
        shape = (self.Hq, self.Hkv, self.hd)
        ws = self._ws(pl.pl_attention_shared_workspace_bytes(self.n, 1, *shape, self.most, self.prompt))
        out = torch.zeros(self.n, self.Hq, self.hd, device="cuda", dtype=torch.bfloat16)
        off, sh = i32([0, self.n]), i32([self.prompt])
        pl.pl_attention_shared(*self._cache(), off.data_ptr(), 0, sh.data_ptr(), out.data_ptr(), ws.data_ptr(), self.n, 1, *shape, self.page, self.pages, self.most, self.prompt)
        self.check(out)


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("positions", [1, 40, 700])
def test_one_score_of_all_positions(hd, positions):
    """All weights are alike, whatever the score is."""
    c = PEAK[hd]
    b = Batch(np.full((3, 4), c), [np.full((positions, 2), c)] * 3, hd, 32)
    b.window(positions, 0)
    b.window(max(1, positions // 2), 3)
    if positions >= 40:
        for rows in (3, 12, 20, 40):   # 6, 24, 40 and 80 columns
            Batch(np.full((rows, 4), c), [np.full((positions, 2), c)] * rows, hd, 32, prompt=positions // 32 * 32).shared()


def _levels(rng, c, n, Hkv):
    """Keys around c: c itself here and there, its bf16 neighbours below, its negative, next to nothing."""
    step = 2.0 ** (np.floor(np.log2(c)) - 7)
    k = rng.choice([c - step, c - 2 * step, c / 2, -c, 0.0, 2.0 ** -20], (n, Hkv))
    k[rng.random((n, Hkv)) < 0.02] = c
    return k


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("down", [0, 3, 6, 9, 12, 15, 17, 20, 22, 24])   # queries of 2^-down of the peak: scores from 2^34 to 2^10
@pytest.mark.parametrize("rows", [2, 5, 10, 19])
def test_one_position_of_many(hd, down, rows):
    """The largest score anywhere, large ones of both signs before it, rows and heads of all magnitudes side by side."""
    rng = np.random.default_rng(100 * down + rows + hd)
    c, prompt, Hq, Hkv = PEAK[hd], 1312, 16, 2
    first = _levels(rng, c, prompt, Hkv)
    levels = [np.concatenate([first, _levels(rng, c, int(m), Hkv)]) for m in rng.integers(1, 300, rows)]
    q = c * 2.0 ** -down * rng.choice([1.0, -1.0, 0.5, 0.25, 2.0 ** -20, 0.0], (rows, Hq))
    q[:, 0] = c * 2.0 ** -down
    b = Batch(q, levels, hd, 32, prompt=prompt, seed=rows)
    b.shared()
    b.window(4000, 0, 4000)      # whole contexts, cut into chunks
    b.window(200, 40)


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_scores_that_rise_and_scores_next_to_each_other(hd):
    """A maximum that moves with every run, from far below zero to far above; and one that a single step of 32 bits sets apart from the next."""
    c = PEAK[hd]
    n = 96 * 32
    steps = np.repeat(np.linspace(-c, c, 96), 32)
    k = np.sign(steps) * 2.0 ** np.floor(np.log2(np.abs(steps))) + 0.0
    k[-32:] = c
    for rows in (2, 10, 20):
        q = np.full((rows, 8), c) * np.array([1.0, 1.0, -1.0, 2.0 ** -14, 1.0, 2.0 ** -20, 1.0, 0.0])
        b = Batch(q, [np.stack([k, k[::-1]], 1)] * rows, hd, 32, prompt=n - 32 * 40)
        b.shared()
        b.window(n, 0)
        b.window(500, 100)
    # 255 * 2^9 * (255 and 254) * 2^a: differences of the scores are a few of their steps
    near = np.where(np.arange(1000) % 97 == 13, 255.0, 254.0) * 2.0 ** 8
    for rows in (2, 10):
        b = Batch(np.full((rows, 8), 255.0 * 2.0 ** 7), [np.stack([near, near], 1)] * rows, hd, 64, prompt=960)
        b.shared()
        b.window(1000, 0)
        b.window(300, 64)
