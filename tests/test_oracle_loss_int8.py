"""Pins of the oracle's token log-probabilities, their gradient and the 8-bit product."""
import numpy as np
import pytest

from oracle import int8, loss


def test_logprob_is_log_of_the_normalised_exponentials():
    rng = np.random.default_rng(0)
    h, w = rng.normal(size=(4, 8)), rng.normal(size=(11, 8))
    y, it = np.array([3, -1, 10, 11]), np.array([1.0, 2.0, 0.5, 1.0])
    lp, lse = loss.token_logprob(h, w, y, it)
    for t in (0, 2):
        e = np.exp(it[t] * (w @ h[t]))
        assert np.isclose(lp[t], np.log(e[y[t]] / e.sum())) and np.isclose(lse[t], np.log(e.sum()))
    assert lp[1] == lse[1] == lp[3] == lse[3] == 0
    assert loss.token_logprob(h[:1], w[:1], np.array([0]))[0][0] == 0   # one entry: certain


@pytest.mark.parametrize("it", [None, np.array([1.4, 0.7, 1.0])])
def test_gradient_matches_differences(it):
    rng = np.random.default_rng(1)
    h, w, g = rng.normal(size=(3, 6)), rng.normal(size=(9, 6)), rng.normal(size=3)
    y = np.array([8, -1, 0])
    L = lambda h, w: g @ loss.token_logprob(h, w, y, it)[0]   # noqa: E731
    dh, dw = loss.token_logprob_grad(h, w, y, loss.token_logprob(h, w, y, it)[1], g, it)
    for a, da, f in ((h, dh, lambda x: L(x, w)), (w, dw, lambda x: L(h, x))):
        for i in np.ndindex(*a.shape):
            e = np.zeros_like(a)
            e[i] = 1e-5
            assert abs((f(a + e) - f(a - e)) / 2e-5 - da[i]) < 1e-8
    assert (dh[1] == 0).all()


def test_codes():
    q, s = int8.quantize_rows(np.array([[127, -127, 0.5, 1.5, 2.5], [0, 0, 0, 0, 0], [1, 2, np.inf, 3, 4], [1e-45, 0, 0, 0, 0], [2, -1, 1, 0, 0.5]]))
    assert s[0] == 1 and q[0].tolist() == [127, -127, 0, 2, 2]
    assert s[1] == 0 and not q[1].any()
    assert np.isnan(s[2]) and not q[2].any()
    assert s[3] == 0 and not q[3].any()
    assert s[4] == np.float32(2) / np.float32(127) and q[4].tolist() == [127, -64, 64, 0, 32]   # 63.5 or just beside it: the exact quotient says


def test_product_and_image():
    rng = np.random.default_rng(2)
    xq, wq = rng.integers(-127, 128, (3, 256)).astype(np.int8), rng.integers(-127, 128, (64, 256)).astype(np.int8)
    sx, sw = rng.random(3).astype(np.float32), rng.random(64).astype(np.float32)
    ref = (xq.astype(np.int64) @ wq.astype(np.int64).T) * sx.astype(np.float64)[:, None] * sw.astype(np.float64)[None, :]
    assert np.allclose(int8.product(xq, sx, wq, sw), ref, rtol=3 * 2.0 ** -24, atol=0)
    image = int8.operand_image(wq)
    for r, k in ((0, 0), (1, 0), (33, 17), (63, 255), (5, 64), (40, 130)):
        at = ((k // 128) * 2 + r // 32) * 4096 + ((k // 16 % 4) * 64 + (k // 64 % 2) * 32 + r % 32) * 16 + k % 16
        assert image[at] == wq[r, k]
