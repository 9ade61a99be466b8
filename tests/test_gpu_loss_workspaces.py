"""Token log-probabilities and their gradient (GPU) in workspaces at an odd address, whose aligned part ends where their size does: what lies directly behind
stays as it is."""
import numpy as np
import pytest
import torch

from test_gpu_loss import GUARD, Call, _batch, _check_forward, _check_gradients

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,vocab,d", [(1, 1, 256), (5, 65, 512), (32, 8192, 256), (33, 8193, 256), (64, 257, 768), (65, 1000, 256), (128, 4096, 256), (129, 513, 512),
                                       (256, 2048, 256), (1025, 900, 256), (8193, 200, 256)])
def test_nothing_is_written_behind_a_workspace(n, vocab, d):
    h, w, target, it, rng = _batch(n, vocab, d, n + vocab, masked=0.0)
    c = Call(h, w, target, it)
    whole = [torch.full((1 + size + GUARD,), 255, dtype=torch.uint8, device="cuda") for size in c.sizes]
    c.ws = [t[1:] for t in whole]
    c.forward()
    _check_forward(c, h, w, target, it)
    g = rng.normal(size=n).astype(np.float32)
    lse = c.lse[:n].clone()
    c.backward(lse, torch.from_numpy(g).cuda())
    _check_gradients(c, h, w, target, lse.cpu().numpy().astype(np.float64), g.astype(np.float64), it)
    for t, size in zip(whole, c.sizes):
        assert t.data_ptr() % 256 == 0 and (t[:256] == 255).all() and (t[size:] == 255).all()


def test_the_largest_workspace_does_for_every_smaller_batch():
    """One workspace for both calls, full of NaN before each, and batches that shrink."""
    vocab, d, most = 700, 256, 1100
    h, w, target, it, rng = _batch(most, vocab, d, 3)
    g = rng.normal(size=most).astype(np.float32)
    c = Call(h, w, target, it)
    ws = torch.empty(max(c.sizes), dtype=torch.uint8, device="cuda")
    for n in (1100, 1024, 700, 256, 130, 128, 64, 40, 32, 1):
        c = Call(h[:n], w, target[:n], it[:n])
        c.ws = [ws, ws]
        ws.fill_(255)
        c.forward()
        torch.cuda.synchronize()
        lse = c.lse[:n].clone()
        ws.fill_(255)
        c.backward(lse, torch.from_numpy(g[:n]).cuda())
        c.ws = []
        _check_forward(c, h[:n], w, target[:n], it[:n])
        _check_gradients(c, h[:n], w, target[:n], lse.cpu().numpy().astype(np.float64), g[:n].astype(np.float64), it[:n])
