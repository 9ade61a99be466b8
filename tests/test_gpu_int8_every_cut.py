"""Every kernel and cut that an 8-bit product may take (GPU), against exact sums in 64 bits on the device, bit for bit; and that the sizes here do take them all
(no GPU needed)."""
import pytest
import torch

import paper_2509_19128_amd as pl

TILES = {0: (32, 128), 1: (64, 128), 2: (128, 128), 3: (128, 256), 4: (64, 64), 5: (256, 256)}
GUARD = 512
# M, N, K: rows, channels and k that fill no whole tile, slice or round
CASES = [(5, 4128, 256), (19, 152064, 256), (30, 5152, 27648), (1, 2080, 18944), (1, 4128, 32768),                              # 32 x 128
         (257, 3616, 768), (33, 17952, 768), (129, 2080, 8960), (61, 3616, 18944),                                              # 64 x 128
         (2101, 32, 256), (3001, 3616, 1280), (99, 55328, 1536), (257, 4640, 8192), (2101, 96, 2560), (125, 5152, 27648),       # 128 x 128
         (3001, 4640, 256), (300, 55328, 2560), (120, 37888, 2560), (300, 3616, 18944), (130, 8224, 13824), (65, 17952, 8960),  # 128 x 256
         (65, 32, 256), (33, 20000, 512), (509, 32, 18944), (1, 64, 8448), (70, 1568, 8960),                                    # 64 x 64
         (5000, 32, 256), (3001, 4128, 3584), (1025, 37888, 3840),                                                              # 256 x 256
         (1, 8192, 1536), (2, 8224, 1280), (3, 4128, 7680), (4, 8192, 7680), (2, 8224, 13824),                                  # up to four rows
         (5, 32, 256), (8, 1536, 8448), (16, 1568, 3584), (17, 4096, 2560), (33, 4096, 1792), (47, 2592, 5120), (64, 2080, 256)]


def need(M, N, K):
    """Bytes of a workspace on a 256-byte boundary that the cut of exactly so many rows has a use for."""
    kernel, splits = pl.pl_debug_gemm_int8_plan(M, N, K)
    if kernel == 6:
        return 0
    up = lambda b: (b + 255) // 256 * 256   # noqa: E731
    codes = (M + 31) // 32 * 32 * K if kernel == 7 else M * ((K + 511) // 512 * 512)
    return up(4 * M) + up(codes) + (4 * splits * M * N if splits > 1 else 0)


def cut(M, N, K):
    """kernel, sliced, W by non-temporal loads, tiles in more than one row"""
    kernel, splits = pl.pl_debug_gemm_int8_plan(M, N, K)
    large, alone = N * K > 8 << 20, kernel < 5 and M <= TILES[kernel][0]
    return kernel, splits > 1, large and (kernel == 7 or alone and kernel < 4)


def test_the_cases_take_every_cut():
    taken = {cut(*c) for c in CASES}
    want = {(k, sliced, cold) for k in range(4) for sliced in (False, True) for cold in (False, True)}
    want |= {(4, False, False), (4, True, False), (5, False, False), (6, False, False), (7, False, False), (7, False, True)}
    want -= {(0, True, False)}   # (slices of 32-row tiles are of large matrices only)
    assert want <= taken, want - taken
    assert {(M + 15) // 16 for M, N, K in CASES if cut(M, N, K)[0] == 7} == {1, 2, 3, 4}
    assert {M for M, N, K in CASES if cut(M, N, K)[0] == 6} == {1, 2, 3, 4}
    # more than 64 KiB of LDS in the one launch of few rows
    assert any(cut(M, N, K)[0] == 6 and 256 + 8 * 4096 + M * (K + 16) + 2048 > 65536 for M, N, K in CASES)


def test_a_workspace_holds_every_cut_of_fewer_rows():
    for N, K in {(N, K) for _, N, K in CASES} | {(1536, 8960), (3584, 18944), (5120, 27648), (32, 133120), (152064, 3584)}:
        for M in (*range(1, 130), *range(130, 5000, 61)):
            if M * K < 1 << 31:
                assert need(M, N, K) + 256 <= pl.pl_gemm_int8_workspace_bytes(M, N, K), (M, N, K)


def test_plans_of_what_is_refused():
    for bad in ((0, 64, 512), (3, 48, 512), (3, 64, 384), (1 << 23, 64, 256)):
        with pytest.raises(pl.PlError):
            pl.pl_debug_gemm_int8_plan(*bad)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", CASES)
def test_products_by_every_cut(M, N, K):
    gen = torch.Generator("cuda").manual_seed(M + N + K)
    x = torch.randn((M, K), generator=gen, device="cuda")
    x *= torch.where(torch.rand(K, generator=gen, device="cuda") < 0.01, 20.0, 1.0)
    x = x.bfloat16()
    wq = torch.randint(-127, 128, (N, K), generator=gen, device="cuda", dtype=torch.int8)
    sw = torch.rand(N, generator=gen, device="cuda") + 0.5
    image = wq.reshape(N // 32, 32, K // 128, 2, 4, 16).permute(2, 0, 4, 3, 1, 5).contiguous()
    sx = (x.abs().amax(1).double() / 127).float()
    xq = torch.round(x.double() / sx.double()[:, None]).clamp(-127, 127)
    ref = torch.empty(M, N, device="cuda")
    for n in range(0, N, 8192):
        ref[:, n:n + 8192] = (xq @ wq[n:n + 8192].double().T.contiguous()).float()   # (integers below 2^53: exact)
    ref = ref * sx[:, None] * sw
    # the aligned part of a workspace at an odd address ends where its size does; what lies behind is to stay as it is
    size, used = pl.pl_gemm_int8_workspace_bytes(M, N, K), need(M, N, K)
    ws = torch.full((1 + size + GUARD,), 77, dtype=torch.uint8, device="cuda")
    assert ws.data_ptr() % 256 == 0
    for out in (torch.float32, torch.bfloat16):
        y = torch.full((M * N + GUARD,), -7.0, device="cuda", dtype=out)
        pl.pl_gemm_int8(x.data_ptr(), K, image.data_ptr(), sw.data_ptr(), y.data_ptr(), pl.PL_F32 if out == torch.float32 else pl.PL_BF16, M, N, K, ws.data_ptr() + 1,
                        torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(y[:M * N].reshape(M, N), ref.to(out))
        assert (y[M * N:] == -7).all() and (ws[256 + used:] == 77).all() and (ws[:256] == 77).all()
