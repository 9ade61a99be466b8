"""Products in 8-bit integers (GPU) through the C ABI against the oracle, bit for bit: codes, int32 sums and the two fp32 products of a result
are fixed by the interface's definition, and a bf16 result is that number rounded once."""
import numpy as np
import pytest
import torch

import paper_2509_19128_amd as pl
import synth
from oracle import int8

pytestmark = pytest.mark.gpu
GUARD = 64


def _bf16(a):
    return synth.bf16_round(np.asarray(a, np.float32)).reshape(np.shape(a))


def _dev(a, dtype, pad=0):
    """A device tensor of these values whose rows are pad elements further apart than they are long."""
    t = torch.zeros(a.shape[0], a.shape[1] + pad, dtype=dtype)
    t[:, :a.shape[1]] = torch.from_numpy(np.ascontiguousarray(a))
    return t.cuda()


def quantize(w, dtype=torch.float32, pad=0):
    N, K = w.shape
    src = _dev(w, dtype, pad)
    q = torch.full((N * K + GUARD,), 99, dtype=torch.int8, device="cuda")
    s = torch.full((N + GUARD,), -7.0, device="cuda")
    pl.pl_quantize_int8(src.data_ptr(), pl.PL_F32 if dtype == torch.float32 else pl.PL_BF16, K + pad, q.data_ptr(), s.data_ptr(), N, K, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (q[N * K:] == 99).all() and (s[N:] == -7).all()
    return q[:N * K], s[:N]


def product(x, w_image, sw, N, out=torch.float32, pad=0, ws=None):
    M, K = x.shape
    xd = _dev(x, torch.bfloat16, pad)
    y = torch.full((M * N + GUARD,), -7.0, device="cuda", dtype=out)
    nbytes = pl.pl_gemm_int8_workspace_bytes(M, N, K)
    ws = torch.full((nbytes + GUARD,), 77, dtype=torch.uint8, device="cuda") if ws is None else ws
    pl.pl_gemm_int8(xd.data_ptr(), K + pad, w_image.data_ptr(), sw.data_ptr(), y.data_ptr(), pl.PL_F32 if out == torch.float32 else pl.PL_BF16,
                    M, N, K, ws.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (y[M * N:] == -7).all() and (ws[nbytes:] == 77).all()
    return y[:M * N].reshape(M, N)


def _same(got, ref):
    ref = torch.from_numpy(ref)
    got = got.cpu()
    if got.dtype == torch.bfloat16:
        ref = ref.to(torch.bfloat16)
    assert torch.equal(got.isnan(), ref.isnan())
    assert torch.equal(got.nan_to_num(0.0), ref.nan_to_num(0.0)), (got.double() - ref.double()).abs().max()


def _inputs(rng, M, N, K):
    x = rng.normal(size=(M, K)) * np.where(rng.random(K) < 0.02, 20.0, 1.0)
    return _bf16(x), (rng.normal(size=(N, K)) * 0.02).astype(np.float32)


@pytest.mark.parametrize("dtype,pad", [("f32", 0), ("bf16", 0), ("f32", 12), ("bf16", 8)])
@pytest.mark.parametrize("N,K", [(32, 256), (96, 768), (64, 4096), (32, 20480)])
def test_codes_and_scales_of_weights(N, K, dtype, pad):
    rng = np.random.default_rng(N + K)
    w = (rng.normal(size=(N, K)) * np.exp(rng.normal(size=(N, 1)) * 4)).astype(np.float32)
    if dtype == "bf16":
        w = _bf16(w)
    q, s = quantize(w, torch.float32 if dtype == "f32" else torch.bfloat16, pad)
    ref_q, ref_s = int8.quantize_rows(w)
    assert np.array_equal(s.cpu().numpy(), ref_s)
    assert np.array_equal(q.cpu().numpy(), int8.operand_image(ref_q))


@pytest.mark.parametrize("dtype,pad", [("f32", 4), ("bf16", 0)])
@pytest.mark.parametrize("N,K", [(4096, 256), (2048, 1792), (64, 8960), (4096, 7424), (32, 14592), (64, 28672), (4096, 20480), (32, 40960), (32, 41216), (96, 57344), (32, 57600)])
def test_codes_of_every_row_length(N, K, dtype, pad):
    rng = np.random.default_rng(N + K)
    w = (rng.normal(size=(N, K)) * 0.02).astype(np.float32)
    w[N // 2, K - 1], w[N - 1, 0], w[3] = 1.5, -np.inf, 0.0
    if dtype == "bf16":
        w = _bf16(w).astype(np.float32)
    q, s = quantize(w, torch.float32 if dtype == "f32" else torch.bfloat16, pad)
    ref_q, ref_s = int8.quantize_rows(w)
    _same(s, ref_s)
    assert np.array_equal(q.cpu().numpy(), int8.operand_image(ref_q).reshape(-1))


def test_codes_of_hard_rows():
    """Ties (to even), the largest and smallest numbers, zeros, infinities and NaN."""
    rng = np.random.default_rng(3)
    w = (rng.normal(size=(32, 256))).astype(np.float32)
    w[0] = np.arange(256) - 127.5                       # scale 128.5 / 127
    w[1] = (np.arange(256) % 255 - 127) * 0.5           # scale 0.5: quotients are integers ...
    w[1, 0] = 63.5
    w[2] = (np.arange(256) % 254 - 126.5) * 2.0         # ... and, with 254 as the largest, halves
    w[2, 5] = 254.0
    w[3] = 0.0
    w[4] = 1e-45 * (np.arange(256) % 120)
    w[5] *= 1e-38
    w[6] *= 1e38 / np.abs(w[6]).max()
    w[7, 3] = np.inf
    w[8, 255] = -np.inf
    w[9, 17] = np.nan
    w[10] = -0.0
    w[11] = 1e-45
    w[12] = np.float32(3.4028235e38)
    w[13] = 2e-37 * rng.normal(size=256)
    q, s = quantize(w)
    ref_q, ref_s = int8.quantize_rows(w)
    assert np.array_equal(s.cpu().numpy(), ref_s, equal_nan=True)
    got = q.cpu().numpy()
    assert np.array_equal(got, int8.operand_image(ref_q))
    assert np.isnan(s.cpu().numpy()[[7, 8, 9]]).all()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [1, 2, 17, 32, 33, 64, 65, 128, 129, 200, 256, 257, 300, 513])
@pytest.mark.parametrize("N,K", [(32, 256), (512, 512), (1056, 768), (288, 1792)])
def test_products_of_every_row_count(M, N, K, out):
    rng = np.random.default_rng(M * 7 + N + K)
    x, w = _inputs(rng, M, N, K)
    wq, sw = int8.quantize_rows(w)
    image = torch.from_numpy(int8.operand_image(wq)).cuda()
    y = product(x, image, torch.from_numpy(sw).cuda(), N, out)
    _same(y, int8.product(*int8.quantize_rows(x), wq, sw))


@pytest.mark.parametrize("M,N,K", [(1, 3584, 3584), (19, 1536, 8960), (64, 17920, 1536), (256, 4608, 3584), (700, 2048, 1536), (3001, 1536, 512), (5, 32, 133120),
                                   (2, 64, 18944), (1500, 544, 5120)])
def test_products_of_decoder_shapes(M, N, K):
    rng = np.random.default_rng(M + N + K)
    x, w = _inputs(rng, M, N, K)
    image, sw = quantize(w)
    wq, ref_sw = int8.quantize_rows(w)
    assert np.array_equal(sw.cpu().numpy(), ref_sw)
    _same(product(x, image, sw, N, torch.bfloat16, pad=8), int8.product(*int8.quantize_rows(x), wq, ref_sw))


def test_largest_sums_do_not_overflow():
    """Rows of +-127 in every place: the largest int32 sum the interface allows."""
    K, N, M = 133120, 32, 3
    x = np.full((M, K), 127.0, np.float32)
    x[1] = -127.0
    w = np.full((N, K), 127.0, np.float32)
    w[5] = -127.0
    image, sw = quantize(w)
    y = product(x, image, sw, N).cpu().numpy()
    ref = np.float32(float(127 * 127 * K)) * np.where(np.arange(M) == 1, -1, 1)[:, None] * np.where(np.arange(N) == 5, -1, 1)[None, :]
    assert np.array_equal(y, ref.astype(np.float32))


def test_a_row_does_not_depend_on_the_others_and_bad_rows_stay_alone():
    rng = np.random.default_rng(11)
    N, K = 640, 1024
    x, w = _inputs(rng, 300, N, K)
    x[7, 100] = np.nan
    x[9, 0] = np.inf
    x[11] = 0.0
    image, sw = quantize(w)
    wq, ref_sw = int8.quantize_rows(w)
    whole = product(x, image, sw, N)
    _same(whole, int8.product(*int8.quantize_rows(x), wq, ref_sw))
    assert whole[7].isnan().all() and whole[9].isnan().all() and (whole[11] == 0).all()
    for rows in ([0], [299, 3], list(range(40, 100))):
        part = product(x[rows], image, sw, N)
        assert torch.equal(part, whole[rows])


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("N,K", [(32, 256), (3584, 1792), (96, 8192), (20000, 512), (64, 16384), (32, 32768)])
def test_few_rows_and_bad_ones_among_them(M, N, K):
    rng = np.random.default_rng(M + N + K)
    x, w = _inputs(rng, M, N, K)
    x[M - 1, K - 1] = np.inf
    if M > 2:
        x[0] = 0.0
        x[1] *= 1e-30
    wq, sw = int8.quantize_rows(w)
    # scales at any place that a float may have
    scales = torch.zeros(N + 1, device="cuda")
    scales[1:] = torch.from_numpy(sw)
    for out in (torch.float32, torch.bfloat16):
        _same(product(_bf16(x), torch.from_numpy(int8.operand_image(wq)).cuda(), scales[1:], N, out), int8.product(*int8.quantize_rows(_bf16(x)), wq, sw))


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [5, 16, 17, 33, 49, 64])
@pytest.mark.parametrize("N,K", [(4096, 2560), (4096, 6912), (4128, 2560)])
def test_narrow_outputs_of_large_weights(M, N, K, out):
    rng = np.random.default_rng(M + N + K)
    x, w = _inputs(rng, M, N, K)
    x[M // 2, 3] = np.nan
    wq, sw = int8.quantize_rows(w)
    scales = torch.from_numpy(sw).cuda()
    _same(product(_bf16(x), torch.from_numpy(int8.operand_image(wq)).cuda(), scales, N, out, pad=8), int8.product(*int8.quantize_rows(_bf16(x)), wq, sw))


@pytest.mark.parametrize("M,K", [(5, 7936), (6, 8192), (70, 8448), (7, 32768), (130, 33024), (5, 33280), (9, 65536)])
def test_rows_that_lanes_hold_and_longer_ones(M, K):
    rng = np.random.default_rng(M + K)
    x, w = _inputs(rng, M, 64, K)
    x[1, K - 1], x[2, 0], x[3] = 300.0, np.inf, 0.0
    wq, sw = int8.quantize_rows(w)
    _same(product(_bf16(x), torch.from_numpy(int8.operand_image(wq)).cuda(), torch.from_numpy(sw).cuda(), 64, pad=16), int8.product(*int8.quantize_rows(_bf16(x)), wq, sw))


def test_millions_of_channels():
    """One row against a W whose turns behind K would lie beyond 32 bits: equal to the same row in a call of five, which takes other kernels."""
    N, K = 2560000, 256
    rng = np.random.default_rng(5)
    x = _bf16(rng.normal(size=(5, K)))
    image = torch.randint(-127, 128, (N * K,), device="cuda", dtype=torch.int8)
    sw = torch.rand(N, device="cuda")
    assert torch.equal(product(x[:1], image, sw, N)[0], product(x, image, sw, N)[0])


def test_replays_of_a_captured_product_with_eager_calls_between():
    rng = np.random.default_rng(12)
    M, N, K = 24, 3584, 1536
    x, w = _inputs(rng, M, N, K)
    other, _ = _inputs(rng, M, N, K)
    image, sw = quantize(w)
    ws = torch.empty(pl.pl_gemm_int8_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    xd = _dev(x, torch.bfloat16)
    y = torch.empty(M, N, device="cuda")
    call = lambda a, out, w_s: pl.pl_gemm_int8(a.data_ptr(), K, image.data_ptr(), sw.data_ptr(), out.data_ptr(), pl.PL_F32, M, N, K, w_s.data_ptr(),  # noqa: E731
                                               torch.cuda.current_stream().cuda_stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(xd, y, ws)
    wq, ref_sw = int8.quantize_rows(w)
    ref = {0: int8.product(*int8.quantize_rows(x), wq, ref_sw), 1: int8.product(*int8.quantize_rows(other), wq, ref_sw)}
    ws2, y2 = torch.empty_like(ws), torch.empty_like(y)
    for i in range(5):
        xd.copy_(torch.from_numpy(other if i & 1 else x))
        y.fill_(-1)
        graph.replay()
        call(_dev(x, torch.bfloat16), y2, ws2)
        torch.cuda.synchronize()
        _same(y, ref[i & 1])
        _same(y2, ref[0])


@pytest.mark.parametrize("N,K", [(512, 256), (3584, 3584)])
def test_graphs_of_every_cut_share_a_workspace_at_an_odd_address(N, K):
    rng = np.random.default_rng(14)
    x, w = _inputs(rng, 600, N, K)
    image, sw = quantize(w)
    ref = int8.product(*int8.quantize_rows(x), *int8.quantize_rows(w))
    xd = _dev(x, torch.bfloat16)
    ws = torch.empty(pl.pl_gemm_int8_workspace_bytes(600, N, K) + 3 + max(pl.pl_gemm_int8_workspace_bytes(m, N, K) for m in (2, 24, 200)), dtype=torch.uint8, device="cuda")
    calls = []
    for M in (2, 24, 200, 600):
        y, graph = torch.empty(M, N, device="cuda", dtype=torch.bfloat16), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pl.pl_gemm_int8(xd.data_ptr(), K, image.data_ptr(), sw.data_ptr(), y.data_ptr(), pl.PL_BF16, M, N, K, ws.data_ptr() + 3, torch.cuda.current_stream().cuda_stream)
        calls.append((M, y, graph))
    for _ in range(3):
        for M, y, graph in calls:
            ws.fill_(255)
            y.fill_(-1)
            graph.replay()
            torch.cuda.synchronize()
            _same(y, ref[:M])


def test_two_streams_at_once_with_workspaces_of_their_own():
    rng = np.random.default_rng(13)
    M, N, K = 40, 2048, 2048
    x, w = _inputs(rng, 2 * M, N, K)
    image, sw = quantize(w)
    xd = _dev(x, torch.bfloat16)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.empty(pl.pl_gemm_int8_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda") for _ in range(2)]
    y = torch.empty(2 * M, N, device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            pl.pl_gemm_int8(xd[i * M:].data_ptr(), K, image.data_ptr(), sw.data_ptr(), y[i * M:].data_ptr(), pl.PL_F32, M, N, K, ws[i].data_ptr(), s.cuda_stream)
    torch.cuda.synchronize()
    _same(y, int8.product(*int8.quantize_rows(x), *int8.quantize_rows(w)))
