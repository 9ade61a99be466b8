"""One workspace, of the size for a program's largest attention, for its smaller ones: nothing behind it is written, and results are those of a workspace of their own."""
import numpy as np
import pytest
import torch

import paper_2509_19128_amd as pl

from paged_util import i32

pytestmark = pytest.mark.gpu

PAGE, BEHIND = 64, 16 << 20


class Cache:
    """Rows that all read the same pages, contexts of their own."""

    def __init__(self, rows, heads, positions):
        g = torch.Generator(device="cuda").manual_seed(4)
        self.heads, self.pages = heads, -(-positions // PAGE)
        Hq, Hkv, hd = heads
        self.pool = torch.randn(self.pages * Hkv * 2 * PAGE * hd, generator=g, device="cuda").to(torch.bfloat16)
        self.q = torch.randn(rows, Hq, hd, generator=g, device="cuda").to(torch.bfloat16)
        self.table = i32(np.tile(np.arange(self.pages), (rows, 1)))
        self.ctx = i32(np.concatenate([[positions], np.random.default_rng(rows).integers(1, positions + 1, rows - 1)]))

    def window(self, ws, n, most, window, sinks):
        out = torch.full_like(self.q[:n], -768.0)
        pl.pl_attention_window(self.q.data_ptr(), self.pool.data_ptr(), self.table.data_ptr(), self.ctx.data_ptr(), out.data_ptr(), ws.data_ptr(), n, *self.heads, PAGE, self.pages, most,
                               window, sinks)
        torch.cuda.synchronize()
        return out.view(torch.int16)

    def shared(self, ws, n, groups, most, shared):
        out = torch.full_like(self.q[:n], -768.0)
        off, lens = i32(np.linspace(0, n, groups + 1).astype(int)), i32([shared // 2] * (groups - 1) + [shared])
        pl.pl_attention_shared(self.q.data_ptr(), self.pool.data_ptr(), self.table.data_ptr(), self.ctx.data_ptr(), off.data_ptr(), 0, lens.data_ptr(), out.data_ptr(), ws.data_ptr(), n, groups,
                               *self.heads, PAGE, self.pages, most, shared)
        torch.cuda.synchronize()
        return out.view(torch.int16)


def _one_for_all(size, largest, calls, run):
    nbytes = size(*largest)
    one = torch.full((nbytes + BEHIND,), 0xA5, device="cuda", dtype=torch.uint8)
    for call in [largest, *calls]:
        assert size(*call) <= nbytes, call
        got = run(one, call)
        assert bool((one[nbytes:] == 0xA5).all()), call
        own = torch.full((size(*call),), 0x3C, device="cuda", dtype=torch.uint8)
        assert torch.equal(got, run(own, call)), call


@pytest.mark.parametrize("heads,largest,calls", [
    ((28, 4, 128), (256, 8192, 4096, 4), [(89, 8192, 4096, 4), (65, 8192, 4096, 4), (31, 8192, 4096, 4), (16, 4096, 4096, 4), (3, 8192, 8192, 0), (70, 8192, 3000, 0)]),
    ((28, 4, 128), (32, 8192, 4096, 4), [(31, 8192, 4096, 4), (9, 8192, 8000, 4), (16, 4096, 4096, 0)]),
    ((8, 2, 32), (700, 20000, 20000, 40), [(160, 20000, 9000, 3), (130, 20000, 20000, 0), (64, 12000, 12000, 0), (1, 20000, 20000, 0)])])
def test_windows(heads, largest, calls):
    c = Cache(largest[0], heads, largest[1])
    _one_for_all(lambda n, most, window, sinks: pl.pl_attention_window_workspace_bytes(n, *heads, most, window, sinks), largest, calls, lambda ws, call: c.window(ws, *call))


@pytest.mark.parametrize("heads,largest,calls", [
    ((28, 4, 128), (128, 8, 9000, 2048), [(100, 8, 9000, 2048), (64, 1, 9000, 2048), (17, 3, 8000, 2000), (2, 1, 9000, 2048), (1, 1, 300, 1), (128, 1, 9000, 2048)]),
    ((10, 2, 64), (128, 128, 30000, 16384), [(128, 1, 30000, 16384), (20, 1, 30000, 16384), (64, 2, 30000, 64), (5, 5, 20000, 0)]),
    ((16, 1, 32), (64, 1, 40000, 40000), [(63, 1, 40000, 40000), (9, 1, 40000, 39000), (8, 4, 40000, 40000)])])
def test_shared_prompts(heads, largest, calls):
    c = Cache(largest[0], heads, largest[2])
    _one_for_all(lambda n, groups, most, shared: pl.pl_attention_shared_workspace_bytes(n, groups, *heads, most, shared), largest, calls, lambda ws, call: c.shared(ws, *call))
