"""Token log-probabilities and their gradient (GPU) through the C ABI against the oracle in 64 bits.

Tolerances, from the arithmetic.  A logit is a sum of d products in fp32, exact before they are added: it is off by at most
e_z = inv_t (d + 2) 2^-24 sum_k |h w|.  lse adds exponentials of fp32 arguments, each off by a few last places of its argument and result
(2^-21 relative where it counts), in sums of at most 64, then groups: e_lse = max e_z + 2^-19 + 2^-23 |lse|.  G is rounded to bf16 (2^-8 relative)
from a probability that is off by (e_z + 2^-20) relative; products and sums as above; a result is rounded to bf16 (2^-8)."""
import numpy as np
import pytest
import torch

import paper_2509_19128_amd as pl
import synth
from oracle import importance, int8, loss

pytestmark = pytest.mark.gpu
GUARD = 64


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _dev(a, pad=0, fill=float("nan")):
    """bf16 rows pad elements further apart than they are long (what lies between is NaN)."""
    if isinstance(a, torch.Tensor):
        return a
    t = torch.full((a.shape[0], a.shape[1] + pad), fill, dtype=torch.bfloat16)
    t[:, :a.shape[1]] = torch.from_numpy(np.ascontiguousarray(a))
    return t.cuda()


class Call:
    """Device copies of one batch, guarded outputs, and the two calls on them."""

    def __init__(self, h, w, target, it=None, pad=0):
        self.n, self.d, self.vocab, self.ld = len(h), h.shape[1], len(w), h.shape[1] + pad
        self.h, self.w = _dev(h, pad), _dev(w, pad)
        self.target = target if isinstance(target, torch.Tensor) else torch.from_numpy(np.asarray(target, np.int32)).cuda()
        self.it = None if it is None else torch.from_numpy(np.asarray(it, np.float32)).cuda()
        self.args = (self.h.data_ptr(), self.ld, self.w.data_ptr(), self.ld, self.target.data_ptr(), 0 if it is None else self.it.data_ptr())
        self.shape = (self.n, self.vocab, self.d)
        self.logprob, self.lse = (torch.full((self.n + GUARD,), -7.0, device="cuda") for _ in range(2))
        self.dh = torch.full((self.n * self.d + GUARD,), -7.0, device="cuda", dtype=torch.bfloat16)
        self.dw = torch.full((self.vocab * self.d + GUARD,), -7.0, device="cuda", dtype=torch.bfloat16)
        self.sizes = pl.pl_token_logprob_workspace_bytes(*self.shape), pl.pl_token_logprob_grad_workspace_bytes(*self.shape)
        # a workspace of NaN (fp32 and bf16 alike): what a call reads there, it has written
        self.ws = [torch.full((b + GUARD,), 255, dtype=torch.uint8, device="cuda") for b in self.sizes]

    def forward(self):
        pl.pl_token_logprob(*self.args, self.logprob.data_ptr(), self.lse.data_ptr(), *self.shape, self.ws[0].data_ptr(), _stream())

    def backward(self, lse, g, dh=True, dw=True):
        pl.pl_token_logprob_grad(*self.args, lse.data_ptr(), g.data_ptr(), self.dh.data_ptr() if dh else 0, self.dw.data_ptr() if dw else 0, *self.shape,
                                 self.ws[1].data_ptr(), _stream())

    def guards(self):
        for t, k in ((self.logprob, self.n), (self.lse, self.n), (self.dh, self.n * self.d), (self.dw, self.vocab * self.d)):
            assert (t[k:] == -7).all()
        for t, k in zip(self.ws, self.sizes):
            assert (t[k:] == 255).all()

    def results(self):
        torch.cuda.synchronize()
        self.guards()
        return self.logprob[:self.n].cpu().numpy(), self.lse[:self.n].cpu().numpy()

    def gradients(self):
        torch.cuda.synchronize()
        self.guards()
        return self.dh[:self.n * self.d].reshape(self.n, self.d).float().cpu().numpy(), self.dw[:self.vocab * self.d].reshape(self.vocab, self.d).float().cpu().numpy()


def _batch(n, vocab, d, seed, masked=0.3, lean=8.0):
    rng = np.random.default_rng(seed)
    w = rng.normal(size=(vocab, d)) * (1.2 / np.sqrt(d))
    target = rng.integers(0, vocab, n)
    w = synth.bf16_round(w.astype(np.float32)).reshape(w.shape)
    h = rng.normal(size=(n, d)) + rng.random((n, 1)) * lean * w[target] / 1.44
    h = synth.bf16_round(h.astype(np.float32)).reshape(h.shape)
    target[rng.random(n) < masked] = -1
    it = (1 / (0.7 + 0.3 * rng.random(n))).astype(np.float32)
    return h, w, target, it, rng


def _e_z(h, w, it):
    return it[:, None] * (h.shape[1] + 2) * 2.0 ** -24 * (np.abs(h.astype(np.float64)) @ np.abs(w.astype(np.float64)).T)


def _check_forward(c, h, w, target, it):
    lp, lse = c.results()
    ref_lp, ref_lse = loss.token_logprob(h, w, target, it)
    e_z = _e_z(h, w, np.ones(len(h)) if it is None else it).max(1)
    e_lse = e_z + 2.0 ** -19 + 2.0 ** -23 * np.abs(ref_lse)
    assert (np.abs(lse - ref_lse) <= e_lse).all(), np.abs(lse - ref_lse).max()
    assert (np.abs(lp - ref_lp) <= e_lse + e_z + 2.0 ** -23 * np.abs(ref_lp)).all(), np.abs(lp - ref_lp).max()
    none = (target < 0) | (target >= len(w))
    assert (lp[none] == 0).all() and (lse[none] == 0).all()


def _check_gradients(c, h, w, target, lse, g, it):
    got_h, got_w = c.gradients()
    one = np.ones(len(h)) if it is None else it.astype(np.float64)
    has = (target >= 0) & (target < len(w))
    h64, w64 = np.where(has[:, None], h, 0).astype(np.float64), w.astype(np.float64)
    p = np.where(has[:, None], np.exp(one[:, None] * (h64 @ w64.T) - np.where(has, lse, 0)[:, None]), 0)
    hot = np.zeros_like(p)
    hot[np.nonzero(has)[0], target[has]] = 1
    scale = np.where(has, g * one, 0)[:, None]
    G = scale * (hot - p)
    e_G = np.abs(scale) * p * (_e_z(h64, w, one) + 2.0 ** -20 + 2.0 ** -23 * np.abs(np.where(has, lse, 0))[:, None]) + 2.0 ** -22 * np.abs(scale) * (hot + p) + 2.0 ** -8 * np.abs(G)
    checks = ((got_h, G @ w64, e_G @ np.abs(w64) + (len(w) + 64) * 2.0 ** -24 * (np.abs(G) @ np.abs(w64))),
              (got_w, G.T @ h64, e_G.T @ np.abs(h64) + (len(h) + 64) * 2.0 ** -24 * (np.abs(G).T @ np.abs(h64))))
    assert (got_h[~has] == 0).all()
    for got, ref, e in checks:
        off = np.abs(got - ref) - (e + 2.0 ** -8 * (np.abs(ref) + e) + 1e-38)
        assert off.max() <= 0, (off.max(), np.abs(got - ref).max(), np.abs(ref).max())


SHAPES = [(1, 1, 256), (1, 64, 256), (2, 63, 256), (5, 65, 512), (31, 100, 256), (33, 255, 768), (64, 256, 256), (65, 257, 256), (100, 1000, 512), (128, 513, 256),
          (129, 4096, 256), (256, 777, 256), (257, 1023, 512), (300, 5000, 256), (520, 321, 1024), (1100, 2049, 256), (3, 20000, 256), (70, 9000, 1536)]


@pytest.mark.parametrize("n,vocab,d", SHAPES)
def test_logprob_and_gradient(n, vocab, d):
    h, w, target, it, rng = _batch(n, vocab, d, n + vocab + d, masked=0.0 if n < 3 else 0.3)
    c = Call(h, w, target, it)
    c.forward()
    _check_forward(c, h, w, target, it)
    g = rng.normal(size=n).astype(np.float32)
    lse = c.lse[:n].clone()
    c.backward(lse, torch.from_numpy(g).cuda())
    _check_gradients(c, h, w, target, lse.cpu().numpy().astype(np.float64), g.astype(np.float64), it)


@pytest.mark.parametrize("pad", [8, 24, 512])
def test_rows_apart_and_no_temperatures(pad):
    h, w, target, _, rng = _batch(77, 600, 512, pad)
    c = Call(h, w, target, None, pad)
    c.forward()
    _check_forward(c, h, w, target, None)
    g = rng.normal(size=77).astype(np.float32)
    lse = c.lse[:77].clone()
    c.backward(lse, torch.from_numpy(g).cuda())
    _check_gradients(c, h, w, target, lse.cpu().numpy().astype(np.float64), g.astype(np.float64), None)


@pytest.mark.parametrize("which", ["dh", "dw"])
def test_one_gradient_alone(which):
    h, w, target, it, rng = _batch(90, 700, 256, 5)
    c = Call(h, w, target, it)
    c.forward()
    g = torch.from_numpy(rng.normal(size=90).astype(np.float32)).cuda()
    lse = c.lse[:90].clone()
    c.backward(lse, g)
    both = [t.copy() for t in c.gradients()]
    c.dh.fill_(-7)
    c.dw.fill_(-7)
    c.backward(lse, g, dh=which == "dh", dw=which == "dw")
    got = c.gradients()
    for name, a, b in zip(("dh", "dw"), got, both):
        assert np.array_equal(a, b) if name == which else (a == -7).all()


@pytest.mark.parametrize("what", ["all", "first", "last", "all but one", "beyond"])
def test_positions_without_a_target_whatever_they_hold(what):
    """Padding rows of NaN and infinities, their lse, g and temperature as bad: zeros for them, and no trace in any other result."""
    n, vocab, d = 150, 500, 256
    h, w, target, it, rng = _batch(n, vocab, d, 7, masked=0.0)
    none = {"all": np.ones(n, bool), "first": np.arange(n) < 70, "last": np.arange(n) >= 70, "all but one": np.arange(n) != 99, "beyond": np.arange(n) % 3 == 0}[what]
    target = np.where(none, {"beyond": vocab}.get(what, -1), target)
    if what == "beyond":
        target[0], target[3], target[6] = 2 ** 31 - 1, -2 ** 31, vocab + 1
    g = rng.normal(size=n).astype(np.float32)
    dirty = h.copy()
    dirty[none] = np.where(rng.random((none.sum(), d)) < 0.5, np.nan, np.inf)
    it_dirty, g_dirty = np.where(none, np.nan, it).astype(np.float32), np.where(none, np.inf, g).astype(np.float32)
    c = Call(dirty, w, target, it_dirty)
    c.forward()
    _check_forward(c, h, w, target, it)
    lse = c.lse[:n].clone()
    lse[torch.from_numpy(none).cuda()] = float("nan")
    c.backward(lse, torch.from_numpy(g_dirty).cuda())
    _check_gradients(c, h, w, target, np.where(none, 0, lse.cpu().numpy()).astype(np.float64), g.astype(np.float64), it)
    if what == "all":
        got = c.gradients()
        assert (got[0] == 0).all() and (got[1] == 0).all()


@pytest.mark.parametrize("n", [1, 20, 33, 100, 128, 129, 300])
def test_batches_without_any_target(n):
    h, w, _, it, rng = _batch(n, 700, 256, n)
    c = Call(np.full_like(h, np.nan), w, np.full(n, -1), it)
    c.forward()
    lp, lse = c.results()
    assert (lp == 0).all() and (lse == 0).all()
    c.backward(c.lse[:n].clone(), torch.ones(n, device="cuda"))
    dh, dw = c.gradients()
    assert (dh == 0).all() and (dw == 0).all()


def test_more_positions_than_a_forward_pass_holds():
    n, vocab, d = 9001, 300, 256
    h, w, target, it, rng = _batch(n, vocab, d, 50, masked=0.05)   # (8551 with a target: two passes)
    c = Call(h, w, target, it)
    c.forward()
    _check_forward(c, h, w, target, it)
    g = rng.normal(size=n).astype(np.float32)
    lse = c.lse[:n].clone()
    c.backward(lse, torch.from_numpy(g).cuda())
    _check_gradients(c, h, w, target, lse.cpu().numpy().astype(np.float64), g.astype(np.float64), it)


@pytest.mark.parametrize("n,ldh,ldw", [(20, 1 << 24, 1 << 20), (200, 1 << 23, 1 << 20), (40, 1 << 25, 256), (3, 256, 1 << 20)])
def test_rows_far_apart(n, ldh, ldw):
    """Rows of h and w that lie gigabytes apart: places beyond 32 bits, and pieces of the vocabulary that end where 32 bits do."""
    vocab, d = 1500, 256
    h, w, target, it, rng = _batch(n, vocab, d, 60 + n, masked=0.1)
    c = Call(h, w, target, it)
    far_h, far_w = (torch.empty((len(a) - 1) * ld + d, dtype=torch.bfloat16, device="cuda") for a, ld in ((h, ldh), (w, ldw)))
    far_h.as_strided((n, d), (ldh, 1)).copy_(c.h)
    far_w.as_strided((vocab, d), (ldw, 1)).copy_(c.w)
    c.args = (far_h.data_ptr(), ldh, far_w.data_ptr(), ldw, *c.args[4:])
    c.forward()
    _check_forward(c, h, w, target, it)
    g = rng.normal(size=n).astype(np.float32)
    lse = c.lse[:n].clone()
    c.backward(lse, torch.from_numpy(g).cuda())
    _check_gradients(c, h, w, target, lse.cpu().numpy().astype(np.float64), g.astype(np.float64), it)


def _large(n, vocab, d, some, seed):
    """A batch made on the device, `some` of whose positions have a target, half of those the last entry of the vocabulary."""
    gen = torch.Generator("cuda").manual_seed(seed)
    h = torch.randn((n, d), generator=gen, device="cuda", dtype=torch.bfloat16)
    w = torch.randn((vocab, d), generator=gen, device="cuda", dtype=torch.bfloat16) * (1.2 / d ** 0.5)
    target = torch.randint(0, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32)
    u = torch.rand(n, generator=gen, device="cuda")
    target[u < some / 2] = vocab - 1
    target[u > some] = -1
    target[-1] = vocab - 1
    return Call(h, w, target), torch.randn(n, generator=gen, device="cuda")


def _check_large(c, g=None):
    """_check_forward and _check_gradients on the device, entries of the vocabulary some thousands at a time."""
    torch.cuda.synchronize()
    c.guards()
    has = c.target >= 0
    y, lse, logprob = c.target[has].long(), c.lse[:c.n][has].double(), c.logprob[:c.n][has].double()
    assert (c.lse[:c.n][~has] == 0).all() and (c.logprob[:c.n][~has] == 0).all()
    h = c.h[has].double()
    step = max(1, (1 << 28) // len(h) // 256 * 256)
    sum_z, most, of_target, e_z = torch.zeros_like(lse), torch.full_like(lse, -float("inf")), torch.zeros_like(lse), torch.zeros_like(lse)
    if g is not None:
        g = g[has].double()[:, None]
        dh, e_dh, G_w = (torch.zeros_like(h) for _ in range(3))
        got_w = c.dw[:c.vocab * c.d].reshape(c.vocab, c.d)

    def close(got, ref, e):
        off = (got.double() - ref).abs() - (e + 2.0 ** -8 * (ref.abs() + e) + 1e-38)
        assert off.max().item() <= 0, off.max().item()
    for v in range(0, c.vocab, step):
        w = c.w[v:v + step].double()
        z, e = h @ w.T, (c.d + 2) * 2.0 ** -24 * (h.abs() @ w.abs().T)
        top = torch.maximum(most, z.max(1).values)
        sum_z = sum_z * (most - top).exp() + (z - top[:, None]).exp().sum(1)
        most, e_z = top, torch.maximum(e_z, e.max(1).values)
        hot = torch.arange(v, v + len(w), device="cuda")[None] == y[:, None]
        of_target += torch.where(hot, z, torch.zeros_like(z)).sum(1)
        if g is not None:
            p = (z - lse[:, None]).exp()
            G = g * (hot.double() - p)
            e_G = g.abs() * p * (e + 2.0 ** -20 + 2.0 ** -23 * lse.abs()[:, None]) + 2.0 ** -22 * g.abs() * (hot + p) + 2.0 ** -8 * G.abs()
            dh += G @ w
            e_dh += e_G @ w.abs()
            G_w += G.abs() @ w.abs()
            close(got_w[v:v + step], G.T @ h, e_G.T @ h.abs() + (len(h) + 64) * 2.0 ** -24 * (G.abs().T @ h.abs()))
    ref = most + sum_z.log()
    e_lse = e_z + 2.0 ** -19 + 2.0 ** -23 * ref.abs()
    assert ((lse - ref).abs() <= e_lse).all()
    assert ((logprob - (of_target - ref)).abs() <= e_lse + e_z + 2.0 ** -23 * (of_target - ref).abs()).all()
    if g is not None:
        got_h = c.dh[:c.n * c.d].reshape(c.n, c.d)
        assert (got_h[~has] == 0).all()
        close(got_h[has], dh, e_dh + (c.vocab + 64) * 2.0 ** -24 * G_w)


@pytest.mark.parametrize("n,vocab,d,some", [(400001, 600, 256, 1.0), (400001, 300, 256, 0.5), (1000, 500, 65536, 0.9), (16, 1000, 65536, 1.0), (3, 1 << 24, 256, 1.0),
                                            (2000, 300000, 256, 0.7), (1000, 65536, 16384, 1.0)])
def test_large_batches_and_gradients(n, vocab, d, some):
    c, g = _large(n, vocab, d, some, n + vocab)
    c.forward()
    c.backward(c.lse[:n].clone(), g)
    _check_large(c, g)


def test_the_most_positions():
    n = 1 << 24
    gen = torch.Generator("cuda").manual_seed(1)
    h = torch.randn((n, 256), generator=gen, device="cuda", dtype=torch.bfloat16)
    w = torch.randn((40, 256), generator=gen, device="cuda", dtype=torch.bfloat16) * 0.1
    target = torch.randint(-3000, 40, (n,), generator=gen, device="cuda", dtype=torch.int32).clamp_(min=-1)
    target[-1] = 39
    logprob, lse = (torch.full((n + GUARD,), -7.0, device="cuda") for _ in range(2))
    ws = torch.empty(pl.pl_token_logprob_workspace_bytes(n, 40, 256), dtype=torch.uint8, device="cuda")
    pl.pl_token_logprob(h.data_ptr(), 256, w.data_ptr(), 256, target.data_ptr(), 0, logprob.data_ptr(), lse.data_ptr(), n, 40, 256, ws.data_ptr(), _stream())
    torch.cuda.synchronize()
    has = target >= 0
    z = h[has].double() @ w.double().T
    e_z = 258 * 2.0 ** -24 * (h[has].double().abs() @ w.double().abs().T).max(1).values
    ref = z.logsumexp(1)
    e_lse = e_z + 2.0 ** -19 + 2.0 ** -23 * ref.abs()
    ref_lp = z.gather(1, target[has].long()[:, None])[:, 0] - ref
    assert ((lse[:n][has] - ref).abs() <= e_lse).all()
    assert ((logprob[:n][has] - ref_lp).abs() <= e_lse + e_z + 2.0 ** -23 * ref_lp.abs()).all()
    assert (lse[:n][~has] == 0).all() and (logprob[:n][~has] == 0).all() and (lse[n:] == -7).all() and (logprob[n:] == -7).all()


def test_temperatures_of_zero_and_below():
    """A zero makes all tokens equally likely; what is no temperature gives its position NaN and no other."""
    n, vocab, d = 30, 500, 256
    h, w, target, it, _ = _batch(n, vocab, d, 70, masked=0.0)
    it[3], it[4], it[5] = 0.0, -1.0, np.nan
    c = Call(h, w, target, it)
    c.forward()
    lp, lse = c.results()
    bad = np.isin(np.arange(n), (4, 5))
    assert np.isnan(lp[bad]).all() and np.isnan(lse[bad]).all() and np.isfinite(lp[~bad]).all()
    assert abs(lp[3] + np.log(vocab)) < 1e-5


@pytest.mark.parametrize("n", [20, 100, 300])
def test_infinite_temperatures_give_nan_and_leave_the_other_positions(n):
    h, w, target, it, _ = _batch(n, 500, 256, 75 + n, masked=0.0)
    it[7], it[n - 1] = np.inf, -np.inf
    c = Call(h, -np.abs(w) if n == 100 else w, target, it)
    c.forward()
    bad = np.isin(np.arange(n), (7, n - 1))
    for r in c.results():
        assert np.isnan(r[bad]).all() and np.isfinite(r[~bad]).all()
    c.backward(c.lse[:n].clone(), torch.ones(n, device="cuda"))
    dh, dw = c.gradients()
    assert np.isnan(dh[bad]).all() and np.isfinite(dh[~bad]).all() and np.isnan(dw).any()


@pytest.mark.parametrize("n", [1, 30, 60, 100, 300])
@pytest.mark.parametrize("vocab", [1, 500, 512])
def test_inverse_temperatures_of_zero(n, vocab):
    h, w, target, it, rng = _batch(n, vocab, 256, 80 + n + vocab, masked=0.0)
    it[::3] = 0.0
    c = Call(h, w, target, it)
    c.forward()
    _check_forward(c, h, w, target, it)
    g = rng.normal(size=n).astype(np.float32)
    lse = c.lse[:n].clone()
    c.backward(lse, torch.from_numpy(g).cuda())
    _check_gradients(c, h, w, target, lse.cpu().numpy().astype(np.float64), g.astype(np.float64), it)
    assert (c.gradients()[0][::3] == 0).all()


def test_a_position_does_not_depend_on_the_others():
    n, vocab, d = 400, 3000, 512
    h, w, target, it, _ = _batch(n, vocab, d, 21)
    c = Call(h, w, target, it)
    c.forward()
    whole = c.results()
    h[5], h[50] = np.nan, np.inf            # bad rows with a target: only their own results are bad
    target[5] = target[50] = 3
    for rows in ([0], [399, 2, 5], list(range(40, 110)), list(range(0, 400, 2)), list(range(400))):
        p = Call(h[rows], w, target[rows], it[rows])
        p.forward()
        got = p.results()
        for a, b in zip(got, whole):
            for i, r in enumerate(rows):
                assert np.isnan(a[i]) if r in (5, 50) else a[i] == b[r], (rows[:3], r)


def test_far_logits():
    """Logits of +-2e4: a certain token, an impossible one (log-prob far below any exponential), all equal ones."""
    n, vocab, d = 40, 1500, 256
    h, w, target, it, rng = _batch(n, vocab, d, 22, masked=0.0)
    h[:20] = synth.bf16_round((h[:20] * 4000).astype(np.float32)).reshape(20, d)
    h[20] = 0
    z = it[:, None] * (h.astype(np.float64) @ w.astype(np.float64).T)
    target[:10], target[10:20] = z[:10].argmax(1), z[10:20].argmin(1)
    c = Call(h, w, target, it)
    c.forward()
    _check_forward(c, h, w, target, it)
    lp = c.results()[0]
    assert lp[:10].min() > -60 and lp[10:20].max() < -5000 and abs(lp[20] + np.log(vocab)) < 1e-5
    lse = c.lse[:n].clone()
    g = np.ones(n, np.float32)
    c.backward(lse, torch.from_numpy(g).cuda())
    # (exponentials of logits of 2e4: their e_z is 2 and more, so the formula's bound says nothing there; from row 20 on it does)
    got_h, got_w = c.gradients()
    assert np.isfinite(got_h).all() and np.isfinite(got_w).all()


def test_gradient_against_differences_of_the_log_probs():
    n, vocab, d = 60, 900, 256
    h, w, target, it, rng = _batch(n, vocab, d, 23)
    g = rng.normal(size=n)
    c = Call(h, w, target, it)
    c.forward()
    c.backward(c.lse[:n].clone(), torch.from_numpy(g.astype(np.float32)).cuda())
    dh, dw = c.gradients()
    L = lambda h, w: g @ loss.token_logprob(h, w, target, it)[0]   # noqa: E731
    for got, f, shape in ((dh, lambda e: L(h + e, w), h.shape), (dw, lambda e: L(h, w + e), w.shape)):
        for k in range(6):
            e = rng.normal(size=shape) * 1e-4
            want, have = (f(e) - f(-e)) / 2, float((got.astype(np.float64) * e).sum())
            # two roundings to bf16 of independent sign on what the direction weighs
            assert abs(want - have) <= 6 * 2 * 2.0 ** -8 * np.linalg.norm(got * e) + 1e-6 * abs(want)


def test_results_are_the_same_bits_from_call_to_call_and_replay_from_a_graph():
    n, vocab, d = 333, 2500, 512
    h, w, target, it, rng = _batch(n, vocab, d, 24)
    other = synth.bf16_round((h * 1.25).astype(np.float32)).reshape(h.shape)
    c = Call(h, w, target, it)
    g = torch.from_numpy(rng.normal(size=n).astype(np.float32)).cuda()
    lse = torch.empty(n, device="cuda")

    def both():
        c.forward()
        lse.copy_(c.lse[:n])
        c.backward(lse, g)

    ref = {}
    for i, x in enumerate((h, other)):
        c.h.copy_(_dev(x))
        both()
        ref[i] = [t.copy() for t in (*c.results(), *c.gradients())]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i in (0, 1, 1, 0, 1):
        c.h.copy_(_dev(other if i else h))
        for t in (c.logprob, c.lse, c.dh, c.dw):
            t.fill_(-7)
        graph.replay()
        for a, b in zip((*c.results(), *c.gradients()), ref[i]):
            assert np.array_equal(a, b)
        both()   # eager work between the replays
        for a, b in zip((*c.results(), *c.gradients()), ref[i]):
            assert np.array_equal(a, b)


@pytest.mark.parametrize("n,vocab", [(20, 700), (100, 700), (1500, 150000)])
def test_replays_find_other_targets_and_two_graphs_share_workspaces(n, vocab):
    """Which positions have a target is found out as a replay runs; 1500 positions of 150000 entries take several pieces.  Graphs replayed in turn leave nothing
    in workspaces, at odd addresses here, that the other one would read."""
    d = 256
    batches = []
    calls = [_large(n, vocab, d, 0.9, 5 + i) for i in range(2)]
    lse = [torch.empty(n, device="cuda") for _ in calls]
    raw = [torch.empty(b + 3, dtype=torch.uint8, device="cuda") for b in calls[0][0].sizes]

    def both(i):
        c, g = calls[i]
        pl.pl_token_logprob(*c.args, c.logprob.data_ptr(), c.lse.data_ptr(), *c.shape, raw[0].data_ptr() + 3, _stream())
        lse[i].copy_(c.lse[:n])
        pl.pl_token_logprob_grad(*c.args, lse[i].data_ptr(), g.data_ptr(), c.dh.data_ptr(), c.dw.data_ptr(), *c.shape, raw[1].data_ptr() + 3, _stream())

    gen = torch.Generator("cuda").manual_seed(9)
    for some in (1.0, 0.05, 0.0, 0.6):
        t = torch.randint(0, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32)
        t[torch.rand(n, generator=gen, device="cuda") >= some] = -1
        batches.append(t)
    ref = {}
    for i, (c, _) in enumerate(calls):
        for k, t in enumerate(batches):
            c.target.copy_(t)
            both(i)
            ref[i, k] = [x.clone() for x in (c.logprob, c.lse, c.dh, c.dw)]
            if k in (0, 3) and vocab < 1000:
                _check_large(*calls[i])
    graphs = [torch.cuda.CUDAGraph() for _ in calls]
    for i, graph in enumerate(graphs):
        with torch.cuda.graph(graph):
            both(i)
    for k in (0, 2, 1, 3, 0, 3):
        for i, (c, _) in enumerate(calls):
            c.target.copy_(batches[k])
            for x in (c.logprob[:n], c.lse[:n], c.dh[:n * d], c.dw[:vocab * d]):
                x.fill_(3)
            for w_s in raw:
                w_s.fill_(255)
            graphs[i].replay()
            for a, b in zip((c.logprob, c.lse, c.dh, c.dw), ref[i, k]):
                assert torch.equal(a, b)


@pytest.mark.parametrize("n", [20, 90, 300])
def test_a_bad_position_leaves_the_other_rows_of_dh(n):
    h, w, target, it, rng = _batch(n, 900, 512, 90 + n)
    c = Call(h, w, target, it)
    c.forward()
    g = torch.from_numpy(rng.normal(size=n).astype(np.float32)).cuda()
    lse = c.lse[:n].clone()
    target[3] = c.target[3] = 5
    c.backward(lse, g, dw=False)
    want = c.gradients()[0]
    g[3] = float("nan")
    c.h[3] = float("inf")
    c.backward(lse, g, dw=False)
    got = c.gradients()[0]
    others = np.arange(n) != 3
    assert np.array_equal(got[others], want[others]) and np.isnan(got[3]).all()


def test_two_streams_at_once():
    calls = []
    for i in range(2):
        h, w, target, it, rng = _batch(120 + 50 * i, 2000, 256, 30 + i)
        c = Call(h, w, target, it)
        c.g = torch.from_numpy(rng.normal(size=c.n).astype(np.float32)).cuda()
        c.forward()
        c.saved = c.lse[:c.n].clone()
        c.backward(c.saved, c.g)
        c.ref = [t.copy() for t in (*c.results(), *c.gradients())]
        calls.append((c, torch.cuda.Stream()))
    for _ in range(10):
        for c, s in calls:
            with torch.cuda.stream(s):
                c.forward()
                c.backward(c.saved, c.g)
    for c, _ in calls:
        for a, b in zip((*c.results(), *c.gradients()), c.ref):
            assert np.array_equal(a, b)


def test_decoder_shape_against_64_bits_on_the_device():
    """The 1.5B shape's head, a ragged microbatch; sampled columns of the gradient, errors in the 2-norm: bf16 rounding of G and of the result
    are independent, sqrt(2) / sqrt(3) 2^-8 at most."""
    n, vocab, d = 777, 151936, 1536
    gen = torch.Generator(device="cuda").manual_seed(5)
    w = (torch.randn(vocab, d, generator=gen, device="cuda") * 0.02).bfloat16()
    target = torch.randint(0, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32)
    h = (torch.randn(n, d, generator=gen, device="cuda") + 18 * torch.rand(n, 1, generator=gen, device="cuda") * w[target.long()].float()).bfloat16()
    target[torch.rand(n, generator=gen, device="cuda") < 0.4] = -1
    has = target >= 0
    lp, lse = (torch.empty(n, device="cuda") for _ in range(2))
    ws = torch.empty(max(pl.pl_token_logprob_workspace_bytes(n, vocab, d), pl.pl_token_logprob_grad_workspace_bytes(n, vocab, d)), dtype=torch.uint8, device="cuda")
    args = (h.data_ptr(), d, w.data_ptr(), d, target.data_ptr(), 0)
    pl.pl_token_logprob(*args, lp.data_ptr(), lse.data_ptr(), n, vocab, d, ws.data_ptr(), _stream())
    z = h.double() @ w.double().T
    ref_lse = torch.logsumexp(z, 1)
    ref_lp = z.gather(1, target.clamp(min=0).long()[:, None])[:, 0] - ref_lse
    # sums of d products: d roundings at most of random sign, half a step of the largest logit each, six standard deviations
    e = 6 * 2.0 ** -24 / np.sqrt(3) * np.sqrt(d) * z.abs().max().item() + 2.0 ** -19
    assert (lse - ref_lse)[has].abs().max() < e and (lp - ref_lp)[has].abs().max() < 2 * e
    assert (lp[~has] == 0).all()
    g = torch.randn(n, generator=gen, device="cuda") / n
    dh, dw = torch.empty(n, d, device="cuda", dtype=torch.bfloat16), torch.empty(vocab, d, device="cuda", dtype=torch.bfloat16)
    pl.pl_token_logprob_grad(*args, lse.data_ptr(), g.data_ptr(), dh.data_ptr(), dw.data_ptr(), n, vocab, d, ws.data_ptr(), _stream())
    G = -torch.exp(z - lse.double()[:, None])
    G.scatter_add_(1, target.clamp(min=0).long()[:, None], torch.ones(n, 1, device="cuda", dtype=torch.float64))
    G *= torch.where(has, g.double(), 0.0)[:, None]
    for got, ref in ((dh, G @ w.double()), (dw, G.T @ h.double())):
        assert (torch.linalg.norm(got.double() - ref) / torch.linalg.norm(ref)).item() < np.sqrt(2 / 3) * 2.0 ** -8


def test_rollout_in_8_bits_and_a_gradient_step():
    """The operators together as the Actor loop uses them: an int8 head samples tokens and records log mu, the bf16 head gives log pi of the same
    tokens, the truncated weights and advantages make g, the gradient updates the head, and the new head is quantised for the next step."""
    m = synth.CONFIGS["tiny"]
    n, vocab, d = 48, m.vocab, m.d_model
    rng = np.random.default_rng(40)
    w = synth.bf16_round((rng.normal(size=(vocab, d)) * 0.05).astype(np.float32)).reshape(vocab, d)
    h = synth.bf16_round(rng.normal(size=(n, d)).astype(np.float32)).reshape(n, d)
    wd, hd = _dev(w), _dev(h)
    wq, sw = torch.empty(vocab * d, dtype=torch.int8, device="cuda"), torch.empty(vocab, device="cuda")
    logits = torch.empty(n, vocab, device="cuda")
    it = torch.ones(n, device="cuda")
    token = torch.empty(n, dtype=torch.int32, device="cuda")
    mu, pi, lse, wt = (torch.empty(n, device="cuda") for _ in range(4))
    sid, pos = torch.arange(n, dtype=torch.int64, device="cuda"), torch.full((n,), 9, dtype=torch.int32, device="cuda")
    forced = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def quantised_logits():
        pl.pl_quantize_int8(wd.data_ptr(), pl.PL_BF16, d, wq.data_ptr(), sw.data_ptr(), vocab, d, _stream())
        pl.pl_gemm_int8(hd.data_ptr(), d, wq.data_ptr(), sw.data_ptr(), logits.data_ptr(), pl.PL_F32, n, vocab, d, ws.data_ptr(), _stream())

    quantised_logits()
    codes = int8.quantize_rows(w)
    assert np.array_equal(logits.cpu().numpy(), int8.product(*int8.quantize_rows(h), *codes))
    pl.pl_sample(logits.data_ptr(), n, vocab, sid.data_ptr(), pos.data_ptr(), it.data_ptr(), forced.data_ptr(), 5, token.data_ptr(), mu.data_ptr(), ws.data_ptr(), _stream())
    pl.pl_token_logprob(hd.data_ptr(), d, wd.data_ptr(), d, token.data_ptr(), it.data_ptr(), pi.data_ptr(), lse.data_ptr(), n, vocab, d, ws.data_ptr(), _stream())
    offs = torch.tensor([0, 20, n], dtype=torch.int64, device="cuda")
    sums, ess, tot = (torch.empty(k, device="cuda", dtype=torch.float64) for k in (4, 2, 3))
    pl.pl_is_ess(pi.data_ptr(), mu.data_ptr(), offs.data_ptr(), 2, 5.0, wt.data_ptr(), sums.data_ptr(), ess.data_ptr(), tot.data_ptr(), _stream())
    y = token.cpu().numpy()
    ref_pi, ref_lse = loss.token_logprob(h, w, y)
    assert np.abs(pi.cpu().numpy() - ref_pi).max() < 2e-5
    w_ref, _, _ = importance.packed_is_ess(pi.cpu().numpy(), mu.cpu().numpy(), offs.cpu().numpy(), 5.0)
    assert np.allclose(wt.cpu().numpy(), w_ref, rtol=1e-6, atol=0) and tot[2].item() > 0.99   # (the policies differ by their rounding only)
    adv = torch.from_numpy(rng.normal(size=n).astype(np.float32)).cuda()
    g = wt * adv / n
    dh, dw = torch.empty(n, d, device="cuda", dtype=torch.bfloat16), torch.empty(vocab, d, device="cuda", dtype=torch.bfloat16)
    assert pl.pl_token_logprob_grad_workspace_bytes(n, vocab, d) <= ws.numel()
    pl.pl_token_logprob_grad(hd.data_ptr(), d, wd.data_ptr(), d, token.data_ptr(), it.data_ptr(), lse.data_ptr(), g.data_ptr(), dh.data_ptr(), dw.data_ptr(), n, vocab, d,
                             ws.data_ptr(), _stream())
    ref_dh, ref_dw = loss.token_logprob_grad(h, w, y, ref_lse, g.cpu().numpy())
    for got, ref in ((dh, ref_dh), (dw, ref_dw)):
        assert np.linalg.norm(got.float().cpu().numpy() - ref) < np.sqrt(2 / 3) * 2.0 ** -8 * np.linalg.norm(ref)
    wd += 0.5 * dw
    quantised_logits()
    new = wd.float().cpu().numpy()
    assert np.array_equal(logits.cpu().numpy(), int8.product(*int8.quantize_rows(h), *int8.quantize_rows(new)))
