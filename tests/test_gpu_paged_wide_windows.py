"""Windows about as long as contexts may be, over rows most of which see far less: a position more or fewer, which no row sees, changes nothing in how the call is cut."""
import numpy as np
import pytest
import torch

import paper_2509_19128_amd as pl

from paged_util import attend, i32, pages_of

pytestmark = pytest.mark.gpu

PAGE = 64


@pytest.mark.parametrize("n,heads,most", [(8, (16, 8, 32), 32768), (32, (28, 4, 128), 131072), (16, (4, 4, 64), 40000)])
def test_a_window_of_all_but_one_position(n, heads, most):
    Hq, Hkv, hd = heads
    rng, g = np.random.default_rng(n), torch.Generator(device="cuda").manual_seed(n)
    ctx = np.clip(np.exp(rng.normal(6.5, 1.2, n)), 1, 9000).astype(int)
    ctx[3] = 20000
    pages = -(-most // PAGE)
    held = -(-ctx.max() // PAGE)
    pool = torch.randn(held * Hkv * 2 * PAGE * hd, generator=g, device="cuda").to(torch.bfloat16)
    table = i32(np.pad(np.tile(rng.permutation(held), (n, 1)), ((0, 0), (0, pages - held)), constant_values=-1))   # (all rows read the same pages)
    q, cd = torch.randn(n, Hq, hd, generator=g, device="cuda").to(torch.bfloat16), i32(ctx)
    outs = []
    for window in (most, most - 1, (most + 20000) // 2):
        ws = torch.empty(pl.pl_attention_window_workspace_bytes(n, Hq, Hkv, hd, most, window, 0), device="cuda", dtype=torch.uint8)
        out = torch.zeros(n, Hq, hd, device="cuda", dtype=torch.bfloat16)
        pl.pl_attention_window(q.data_ptr(), pool.data_ptr(), table.data_ptr(), cd.data_ptr(), out.data_ptr(), ws.data_ptr(), n, Hq, Hkv, hd, PAGE, pages, most, window, 0)
        torch.cuda.synchronize()
        outs.append(out)
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
    k, v = pages_of(pool, table[0, :held].cpu().numpy(), Hkv, hd, PAGE)
    for b in (0, 3, n - 1):
        ref, e = attend(q[b].float().cpu().numpy(), k[:ctx[b]], v[:ctx[b]])
        for out in outs:
            assert (np.abs(out[b].float().cpu().numpy() - ref) <= e).all()
