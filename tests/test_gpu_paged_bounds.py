"""Attention over shared prompts behind bounds far above what rows hold, as a captured step has to pass them: the cut of a prompt goes by its own length."""
import numpy as np
import pytest
import torch

import paper_2509_19128_amd as pl

from paged_util import attend, i32, pages_of

pytestmark = pytest.mark.gpu

PAGE = 64


def _call(heads, prompts, rows, own, most, shared_most, seed=0):
    """Groups of `rows` rows behind prompts of these lengths, `own` positions each behind them; the call's result and its operands."""
    Hq, Hkv, hd = heads
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    n, per = len(prompts) * rows, -(-(max(prompts) + own) // PAGE)
    pages = -(-most // PAGE)
    table, at = np.full((n, pages), -1), 0
    for k, c in enumerate(prompts):
        whole = c // PAGE
        first, at = np.arange(at, at + whole), at + whole
        for b in range(k * rows, k * rows + rows):
            more = -(-(c + own) // PAGE) - whole
            table[b, :whole], table[b, whole:whole + more], at = first, np.arange(at, at + more), at + more
    pool = torch.randn(at * Hkv * 2 * PAGE * hd, generator=g, device="cuda").to(torch.bfloat16)
    q = torch.randn(n, Hq, hd, generator=g, device="cuda").to(torch.bfloat16)
    ctx = np.repeat(prompts, rows) + rng.integers(1, own + 1, n)
    td, cd, off, sh = i32(table), i32(ctx), i32(np.arange(len(prompts) + 1) * rows), i32([c // PAGE * PAGE for c in prompts])
    size = pl.pl_attention_shared_workspace_bytes(n, len(prompts), Hq, Hkv, hd, most, shared_most)
    ws = torch.full((size + 4096,), 0xA5, device="cuda", dtype=torch.uint8)
    out = torch.zeros(n, Hq, hd, device="cuda", dtype=torch.bfloat16)
    pl.pl_attention_shared(q.data_ptr(), pool.data_ptr(), td.data_ptr(), cd.data_ptr(), off.data_ptr(), 0, sh.data_ptr(), out.data_ptr(), ws.data_ptr(), n, len(prompts), Hq, Hkv, hd, PAGE,
                           pages, most, shared_most)
    torch.cuda.synchronize()
    assert bool((ws[size:] == 0xA5).all())
    return out, (q, pool, table[:, :per], ctx)


@pytest.mark.parametrize("heads,prompts,rows", [((40, 8, 128), [16384], 64), ((40, 8, 128), [9000], 16), ((28, 4, 128), [2048, 4096, 700, 1000], 16), ((8, 1, 64), [30000, 64], 20),
                                                ((16, 4, 32), [6000] * 3, 3), ((16, 1, 128), [45000], 512)])   # (the last: chunks of more pages than a wavefront has lanes)
def test_bits_do_not_depend_on_the_bound_of_prompts(heads, prompts, rows):
    n = len(prompts) * rows
    least = max(max(prompts) + 200, (512 << 20) // (n * heads[1] * heads[2] * 4) + 1)   # (a call that shares)
    first, operands = _call(heads, prompts, rows, 200, least, least)
    for most in (131072, 1 << 20):
        assert torch.equal(first.view(torch.int16), _call(heads, prompts, rows, 200, max(most, least), max(most, least))[0].view(torch.int16)), most
    q, pool, table, ctx = operands
    for b in {0, rows, n - 1} & set(range(n)):
        k, v = (a[:ctx[b]] for a in pages_of(pool, table[b, :-(-ctx[b] // PAGE)], heads[1], heads[2], PAGE))
        ref, e = attend(q[b].float().cpu().numpy(), k, v)
        assert (np.abs(first[b].float().cpu().numpy() - ref) <= e).all()


@pytest.mark.parametrize("most,shared_most", [(17584, 16384), (131072, 16384), (131072, 131072), (1 << 20, 16384)])
def test_results_behind_any_bounds(most, shared_most):
    """Long own parts that may be, which ask for few chunks of what is shared, and prompts that leave most of the chunks there is room for unused."""
    heads, prompts, rows = (14, 2, 128), [15000, 40, 3000], 5
    out, (q, pool, table, ctx) = _call(heads, prompts, rows, 300, most, shared_most)
    for b in range(len(ctx)):
        k, v = (a[:ctx[b]] for a in pages_of(pool, table[b, :-(-ctx[b] // PAGE)], heads[1], heads[2], PAGE))
        ref, e = attend(q[b].float().cpu().numpy(), k, v)
        assert (np.abs(out[b].float().cpu().numpy() - ref) <= e).all(), b
