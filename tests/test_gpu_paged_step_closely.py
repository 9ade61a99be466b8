"""The steps of test_gpu_paged_step.py looked at closely: after each, every place that a row holds has the key and the value of its own token, and both attentions are within their own
rounding of the softmax over exactly those, so that a token that is lost, twice there or old shows wherever it is."""
import numpy as np
import pytest
import torch

from oracle import paged

from paged_util import HALF, attend, bf16, i32, pages_of
from test_gpu_paged_step import EPS, FREQ, HD, N_PAGES, NEW, PAGE, ROWS, WIDTH, Device, Hkv, Host, Hq, _schedule

pytestmark = pytest.mark.gpu


class Cache(Host):
    """With keys in 64 bits, and how far a bf16 key may be off: fp32 sum of squares, root, quotient, products and angle, 32 roundings of the pair that is turned, then half a step."""

    def __init__(self, pages):
        super().__init__(pages)
        self.K, self.off = np.zeros((N_PAGES * PAGE, Hkv, HD)), np.zeros((N_PAGES * PAGE, Hkv, HD))

    def append(self, x, gq, gk, slot, position):
        k = paged.norm_rope(x[:, Hq:Hq + Hkv], gk, EPS, position, FREQ)
        lo, hi = np.split(np.abs(paged.norm_rope(x[:, Hq:Hq + Hkv], gk, EPS, 0 * position, FREQ)), 2, -1)
        e = 32 * 2.0 ** -24 * np.concatenate([lo + hi, lo + hi], -1)
        used = slot >= 0
        self.K[slot[used]], self.off[slot[used]] = k[used], (e + HALF[torch.bfloat16] * (np.abs(k) + e))[used]
        self.V[slot[used]] = x[used, Hq + Hkv:]


@pytest.mark.parametrize("pages", [12, 5000])   # of a row at most: few enough that nothing is shared, and enough that prompts are
@pytest.mark.parametrize("captured", [False, True])
def test_every_token_is_in_its_place(captured, pages):
    rng = np.random.default_rng(17)
    (gq, gq_d), (gk, gk_d) = (bf16(1 + 0.3 * rng.normal(size=HD)) for _ in range(2))
    host, dev = Cache(pages), Device(gq_d, gk_d, pages)
    owned = np.zeros(ROWS, np.int64)
    graph = None
    if captured:
        dev.step(torch.cuda.current_stream().cuda_stream)   # (nothing wanted: nothing changes)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dev.step(torch.cuda.current_stream().cuda_stream)
    for what in _schedule(rng):
        want = host.len.copy()
        for b, n in what.get("want", {}).items():
            want[b] = n
            if n < owned[b] * PAGE:
                owned[b] = 0
        want[want > 0] += what.get("grow", 0)
        if "fork" in what:
            for lead, rows, n in what["fork"]:
                for b in rows:
                    host.table[b, :n // PAGE] = host.table[lead, :n // PAGE]
                    host.len[b], owned[b], want[b] = n, n // PAGE, n + 5
                owned[lead] = n // PAGE
            dev.table.copy_(i32(host.table))
            dev.len.copy_(i32(host.len))
            dev.shared.copy_(i32([64, 64]))
        if what.get("want", {}).get(5) == 0:   # (row 5 leaves its group)
            dev.group_rows.copy_(i32([2, 0, 0, 1, 3, 6]))
        x, xd = bf16(rng.normal(size=(NEW, WIDTH)))
        dev.x.copy_(xd)
        dev.want.copy_(i32(want))
        dev.owned.copy_(i32(owned))
        dev.out.fill_(-768.0)
        torch.cuda.synchronize()
        if graph is not None:
            graph.replay()
        else:
            dev.step(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        offsets, slot, position, status = host.plan(want, owned)
        assert int(dev.status) == status and np.array_equal(dev.table.cpu().numpy(), host.table)
        host.append(x.reshape(NEW, -1, HD).astype(np.float64), gq.astype(np.float64), gk.astype(np.float64), slot, position)
        K, V = pages_of(dev.pool, np.arange(N_PAGES), Hkv, HD, PAGE)
        last, out = dev.last.float().cpu().numpy(), dev.out.float().cpu().numpy()
        for b in range(ROWS):
            if host.len[b] == 0:
                assert (out[:, b] == -768).all()
                continue
            pos = np.arange(host.len[b])
            at = host.table[b, pos // PAGE] * PAGE + pos % PAGE
            assert (np.abs(K[at] - host.K[at]) <= host.off[at]).all() and np.array_equal(V[at], host.V[at]), b
            see = paged.visible(host.len[b], 50, 3)
            for got, rows in ((out[0, b], at), (out[1, b], at[see])):
                ref, e = attend(last[b], K[rows], V[rows])
                assert (np.abs(got - ref) <= e).all(), (b, np.abs(got - ref).max(), e.max())
