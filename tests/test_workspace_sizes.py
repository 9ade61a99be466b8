"""A workspace for the largest call of a program does for its smaller ones: sizes grow with the number of rows (no GPU needed)."""
import pytest

import paper_2509_19128_amd as pl


def _growing(size, rows):
    last = 0
    for n in rows:
        b = size(n)
        assert b >= last, (n, b, last)
        last = b


ROWS = [*range(1, 700), *range(700, 5000, 37), 5000, 10000, 19200, 19201, 38400, 38401, 50000, 65536]


@pytest.mark.parametrize("N,K", [(32, 256), (32, 133120), (512, 256), (1536, 8960), (1536, 1536), (3584, 3584), (4096, 7168), (4128, 2560), (4608, 3584), (5120, 27648), (3584, 18944),
                                 (17920, 1536), (37888, 3584), (55296, 5120), (152064, 3584), (76800, 1024), (2560000, 256)])
def test_8_bit_products(N, K):
    _growing(lambda M: pl.pl_gemm_int8_workspace_bytes(M, N, K), [M for M in ROWS if M * K < 1 << 31])


@pytest.mark.parametrize("vocab,d", [(1, 256), (4096, 256), (32000, 2048), (152064, 3584), (300000, 65536)])
def test_log_probabilities_and_their_gradient(vocab, d):
    for size in (pl.pl_token_logprob_workspace_bytes, pl.pl_token_logprob_grad_workspace_bytes):
        _growing(lambda n: size(n, vocab, d), [n for n in ROWS if (n + 255) // 256 * 256 * d * 2 < 1 << 31])
