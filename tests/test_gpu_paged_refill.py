"""Rows whose sequences end and that begin others in the same step: one call of the page plan for the ends and one for what is wanted, one by one and captured."""
import numpy as np
import pytest
import torch

import paper_2509_19128_amd as pl
from oracle import paged

from paged_util import i32

pytestmark = pytest.mark.gpu


class Plans:
    def __init__(self, n, pages, page, n_pages, max_new):
        self.shape = (n, page, pages, n_pages, max_new)
        i = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.int32)   # noqa: E731
        self.len, self.want, self.ends, self.owned, self.table = i(n), i(n), i(n), i(n), torch.full((n, pages), -1, device="cuda", dtype=torch.int32)
        self.free, self.count = i32(np.arange(n_pages)[::-1]), i32([n_pages])
        self.offsets, self.slot, self.position, self.status = i(n + 1), i(max_new), i(max_new), i(2, 1)

    def call(self, want, status, stream):
        n, page, pages, n_pages, max_new = self.shape
        pl.pl_kv_plan(self.len.data_ptr(), want.data_ptr(), self.owned.data_ptr(), self.table.data_ptr(), self.free.data_ptr(), self.count.data_ptr(), self.count.data_ptr(),
                      self.len.data_ptr(), self.offsets.data_ptr(), self.slot.data_ptr(), self.position.data_ptr(), status.data_ptr(), n, page, pages, n_pages, max_new, stream)

    def step(self):
        stream = torch.cuda.current_stream().cuda_stream
        self.call(self.ends, self.status[0], stream)
        self.call(self.want, self.status[1], stream)


@pytest.mark.parametrize("n,pages,page,max_new", [(9, 6, 32, 700), (300, 5, 64, 9000), (1500, 4, 32, 30000)])
@pytest.mark.parametrize("captured", [False, True])
def test_rows_that_end_and_begin_in_one_step(n, pages, page, max_new, captured):
    rng = np.random.default_rng(n)
    n_pages, longest = n * pages, pages * page
    d = Plans(n, pages, page, n_pages, max_new)
    graph = None
    if captured:
        d.step()   # (nothing wanted: nothing changes)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            d.step()
    have, table, free, count = np.zeros(n, np.int64), np.full((n, pages), -1), np.arange(n_pages)[::-1].copy(), n_pages
    zero = np.zeros(n, np.int64)
    for _ in range(12):
        over = (rng.random(n) < 0.15) & (have > 0)
        ends = np.where(over, 0, have)
        want = np.where(have > 0, np.minimum(have + 1, longest), 0)
        fresh = (over | (have == 0)) & (rng.random(n) < 0.7)
        want[over] = 0
        want[fresh] = rng.integers(1, longest + 1, int(fresh.sum()))   # shorter and longer than what the row held
        late = np.cumsum(np.maximum(want - ends, 0)) > max_new
        want[late] = ends[late]
        d.ends.copy_(i32(ends))
        d.want.copy_(i32(want))
        torch.cuda.synchronize()
        if graph is None:
            d.step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        table, free, count, mid, _, _, _, s0 = paged.plan(have, ends, zero, table, free, count, page, max_new)
        table, free, count, have, offsets, slot, position, s1 = paged.plan(mid, want, zero, table, free, count, page, max_new)
        assert (s0, s1) == (0, 0) and d.status.flatten().tolist() == [0, 0]
        for name, ref in (("len", want), ("table", table), ("free", free), ("count", [count]), ("offsets", offsets), ("slot", slot), ("position", position)):
            assert np.array_equal(getattr(d, name).cpu().numpy(), ref), name
        for b in np.flatnonzero(fresh & ~late):   # all of a new sequence's tokens are new
            assert list(position[offsets[b]:offsets[b + 1]]) == list(range(want[b]))
        held = [table[b, j] for b in range(n) for j in range(-(-want[b] // page))]
        assert sorted(held + list(free[:count])) == list(range(n_pages))


def test_a_length_that_falls_cuts_a_sequence_short():
    d = Plans(2, 4, 32, 8, 64)
    for want, new in (([100, 3], None), ([64, 4], 1), ([33, 0], 0), ([65, 1], 33)):
        d.want.copy_(i32(want))
        before = d.len.cpu().numpy()
        if max(want) == 100:   # (more new tokens than a call has room for: by two)
            d.want.copy_(i32([50, 3]))
            d.call(d.want, d.status[1], 0)
            d.want.copy_(i32(want))
            torch.cuda.synchronize()
            before = d.len.cpu().numpy()
        table = d.table.cpu().numpy()
        d.call(d.want, d.status[1], 0)
        torch.cuda.synchronize()
        assert int(d.status[1]) == 0 and d.len.tolist() == want
        kept = np.minimum(before, want)
        for b in range(2):
            assert np.array_equal(d.table.cpu().numpy()[b, :-(-kept[b] // 32)], table[b, :-(-kept[b] // 32)])
        if new is not None:
            assert int(d.offsets[2]) == new == int(np.maximum(np.array(want) - before, 0).sum())
