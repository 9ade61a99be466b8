"""What the token log-probabilities and the 8-bit products refuse, before anything is launched (no GPU needed)."""
import pytest

import paper_2509_19128_amd as pl

P = 4096   # an address that nothing reads


def refused(f, *a):
    with pytest.raises(pl.PlError) as e:
        f(*a)
    assert e.value.code == pl.PL_E_INVAL
    return str(e.value)


LOSS = dict(h=P, ldh=512, w=P, ldw=512, target=P, it=0, n=5, vocab=100, d=512)


@pytest.mark.parametrize("bad", [dict(h=0), dict(w=0), dict(target=0), dict(n=0), dict(n=-3), dict(n=(1 << 24) + 1), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(d=0),
                                 dict(d=128, ldh=128, ldw=128), dict(d=500), dict(d=65792, ldh=65792, ldw=65792), dict(ldh=504), dict(ldw=256), dict(ldh=516),
                                 dict(ldw=514), dict(ldw=(1 << 20) + 8), dict(h=P + 8), dict(w=P + 2)])
def test_logprob_and_gradient_refuse(bad):
    a = {**LOSS, **bad}
    first = (a["h"], a["ldh"], a["w"], a["ldw"], a["target"], a["it"])
    refused(pl.pl_token_logprob, *first, P, P, a["n"], a["vocab"], a["d"], P)
    refused(pl.pl_token_logprob_grad, *first, P, P, P, P, a["n"], a["vocab"], a["d"], P)


def test_outputs_and_workspaces_are_needed():
    first = (P, 512, P, 512, P, 0)
    for i in range(2):
        refused(pl.pl_token_logprob, *first, *[0 if i == j else P for j in range(2)], 5, 100, 512, P)
    refused(pl.pl_token_logprob, *first, P, P, 5, 100, 512, 0)
    for lse, g, ws in ((0, P, P), (P, 0, P), (P, P, 0)):
        refused(pl.pl_token_logprob_grad, *first, lse, g, P, P, 5, 100, 512, ws)
    assert "neither" in refused(pl.pl_token_logprob_grad, *first, P, P, 0, 0, 5, 100, 512, P)
    for dh, dw in ((P + 8, P), (P, P + 4)):
        assert "dh and dw" in refused(pl.pl_token_logprob_grad, *first, P, P, dh, dw, 5, 100, 512, P)
    assert "2 GiB" in refused(pl.pl_token_logprob_grad, P, 256, P, 256, P, 0, P, P, P, P, 1 << 22, 100, 256, P)


def test_workspace_sizes_of_what_is_refused_are_zero_and_of_the_rest_are_not():
    for bad in ((0, 100, 512), (5, 0, 512), (5, 100, 100), (5, 100, 1 << 17), (-1, 100, 512)):
        assert pl.pl_token_logprob_workspace_bytes(*bad) == 0 and pl.pl_token_logprob_grad_workspace_bytes(*bad) == 0
    assert pl.pl_token_logprob_grad_workspace_bytes(1 << 22, 100, 256) == 0
    for n, vocab, d in ((1, 1, 256), (4096, 152064, 3584), (100000, 152064, 5120), (1 << 24, 64, 256)):
        assert pl.pl_token_logprob_workspace_bytes(n, vocab, d) > 0
        assert (pl.pl_token_logprob_grad_workspace_bytes(n, vocab, d) > 0) == (n * d * 2 < 1 << 31)
    # a piece of the vocabulary at a time: far below the logits' 2.5 GB
    assert pl.pl_token_logprob_grad_workspace_bytes(4096, 152064, 3584) < 600 << 20
    assert pl.pl_token_logprob_workspace_bytes(4096, 152064, 3584) < 200 << 20


INT8 = dict(x=P, ldx=512, wq=P, sw=P, y=P, yt=1, M=3, N=64, K=512, ws=P)


@pytest.mark.parametrize("bad", [dict(x=0), dict(wq=0), dict(sw=0), dict(y=0), dict(ws=0), dict(yt=2), dict(yt=-1), dict(M=0), dict(M=-1), dict(N=0), dict(N=48), dict(K=0),
                                 dict(K=384), dict(K=133376, ldx=133376), dict(N=32 << 18, K=256), dict(M=1 << 23, K=256), dict(ldx=256), dict(ldx=516), dict(x=P + 8),
                                 dict(wq=P + 1), dict(y=P + 8)])
def test_product_refuses(bad):
    a = {**INT8, **bad}
    refused(pl.pl_gemm_int8, a["x"], a["ldx"], a["wq"], a["sw"], a["y"], a["yt"], a["M"], a["N"], a["K"], a["ws"])
    if set(bad) & {"M", "N", "K"}:
        assert pl.pl_gemm_int8_workspace_bytes(a["M"], a["N"], a["K"]) == 0


@pytest.mark.parametrize("bad", [dict(w=0), dict(q=0), dict(s=0), dict(dtype=2), dict(ldw=256), dict(ldw=516), dict(dtype=1, ldw=514), dict(N=0), dict(N=33), dict(K=128),
                                 dict(K=133376, ldw=133376), dict(N=32 << 18, K=256), dict(w=P + 4), dict(q=P + 8)])
def test_quantisation_refuses(bad):
    a = {**dict(w=P, dtype=0, ldw=512, q=P, s=P, N=64, K=512), **bad}
    refused(pl.pl_quantize_int8, a["w"], a["dtype"], a["ldw"], a["q"], a["s"], a["N"], a["K"])
