"""Timed cases of the trainer-side log-probabilities and of the products in 8-bit integers.

`logprob` and `grad` are the learner's side of the Actor loop: the log-probability of recorded tokens under the current
weights (which the truncated importance weights compare with the recorded one), and its gradient to the hidden states and
the LM head.  `int8` and `update` are the generation side in 8 bits: products of a decode step or a prompt pass with
quantised weights, and an in-flight update that quantises new weights and goes on with the first product.

Shapes are those of the benchmark's decoder configurations (widths 256 to 5120, vocabularies of 4096 to 152064).
"""
from __future__ import annotations

import math

import torch

own = False


# ---- the cases -----------------------------------------------------------------------------------------

def listed():
    return [
        # one optimizer microbatch of the 7B shape: packed sequences, a fifth of the positions are prompts without a target
        dict(name="logprob 7b 4096", kind="logprob", n=4096, vocab=152064, d=3584, masked=0.2),
        # a short sequence scored by itself, 1.5B shape: the head is streamed once
        dict(name="logprob 1.5b 61", kind="logprob", n=61, vocab=151936, d=1536, masked=0.1),
        # the smallest call: a few tokens of the tiny shape (launch latency)
        dict(name="logprob tiny 5", kind="logprob", n=5, vocab=4096, d=256, masked=0.0),
        # the gradient of the same microbatch
        dict(name="grad 7b 4096", kind="grad", n=4096, vocab=152064, d=3584, masked=0.2),
        # a ragged microbatch of the 1.5B shape whose prompts are half of it
        dict(name="grad 1.5b 777", kind="grad", n=777, vocab=151936, d=1536, masked=0.5),
        # the smallest gradient
        dict(name="grad tiny 33", kind="grad", n=33, vocab=4096, d=256, masked=0.1),
        # gate/up of the 7B shape at its benchmark batch
        dict(name="int8 7b gate/up 256", kind="int8", M=256, N=37888, K=3584, out="bf16"),
        # attention output projection of the 7B shape, a decayed batch: latency and the weight stream
        dict(name="int8 7b o 19", kind="int8", M=19, N=3584, K=3584, out="f32"),
        # down projection of the 32B shape in a prompt pass
        dict(name="int8 32b down 3001", kind="int8", M=3001, N=5120, K=27648, out="bf16"),
        # the smallest product
        dict(name="int8 tiny 1", kind="int8", M=1, N=512, K=256, out="f32"),
        # an update of the 7B shape's gate/up weights, bf16 masters, and the first step's product
        dict(name="update 7b gate/up 64", kind="update", M=64, N=37888, K=3584, src="bf16", out="bf16"),
        # the 1.5B shape's down projection from fp32 masters
        dict(name="update 1.5b down 8", kind="update", M=8, N=1536, K=8960, src="f32", out="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST = 4096 * 152064 * 3584   # products of the largest listed logprob and grad


def draw(rng):
    kind = rng.choice(["logprob", "grad", "int8", "update"])
    if kind in ("logprob", "grad"):
        d = 256 * rng.randint(1, 20)
        vocab = min(152064, _log(rng, 1000, 200000))
        n = min(_log(rng, 1, 4096), MOST // (vocab * d))
        return dict(kind=kind, n=n, vocab=vocab, d=d, masked=rng.choice([0.0, 0.1, 0.3, 0.6]))
    K = 256 * _log(rng, 1, 108)
    N = 32 * _log(rng, 4, 1184)
    if kind == "update":
        return dict(kind=kind, M=_log(rng, 1, 256), N=N, K=K, src=rng.choice(["bf16", "f32"]), out=rng.choice(["bf16", "f32"]))
    return dict(kind=kind, M=_log(rng, 1, 3001), N=N, K=K, out=rng.choice(["bf16", "f32"]))


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


# ---- inputs --------------------------------------------------------------------------------------------

def _operand_order(q):
    """[N, K] codes -> the image that the product streams: blocks of 32 rows x 128 columns, column block by column block."""
    n, k = q.shape
    return q.reshape(n // 32, 32, k // 128, 2, 4, 16).permute(2, 0, 4, 3, 1, 5).contiguous().reshape(-1)


def _loss_inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, vocab, d = case["n"], case["vocab"], case["d"]
    w = torch.randn(vocab, d, generator=g, device="cuda", dtype=torch.bfloat16) * 0.02
    target = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    # normed hidden states that lean towards their token, from hardly to clearly: log-probs from about -log(vocab) to 0
    lean = 14.0 * torch.rand(n, 1, generator=g, device="cuda") / (4e-4 * d)
    h = torch.randn(n, d, generator=g, device="cuda") + lean * w[target.long()].float()
    h = h.to(torch.bfloat16)
    if case["masked"]:
        target[torch.rand(n, generator=g, device="cuda") < case["masked"]] = -1
    it = 1.0 / (0.7 + 0.3 * torch.rand(n, generator=g, device="cuda"))
    return dict(h=h, w=w, target=target, it=it), g


def _int8_inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    M, N, K = case["M"], case["N"], case["K"]
    # activations with a few channels far larger than the rest
    x = torch.randn(M, K, generator=g, device="cuda")
    x *= torch.where(torch.rand(K, generator=g, device="cuda") < 0.01, 20.0, 1.0)
    w = torch.randn(N, K, generator=g, device="cuda") * 0.02
    return x.to(torch.bfloat16), w


def prepare(case, seed):
    if case["kind"] in ("logprob", "grad"):
        st, g = _loss_inputs(case, seed)
        n, vocab, d = case["n"], case["vocab"], case["d"]
        st["case"] = case
        if case["kind"] == "logprob":
            st["logprob"], st["lse"] = (torch.empty(n, device="cuda") for _ in range(2))
        else:
            # what the forward pass left: lse, and the loss's gradient to the log-probs (advantage x truncated weight / positions)
            z = (st["h"].float() @ st["w"].float().T) * st["it"][:, None]
            st["lse"] = torch.where(st["target"] >= 0, torch.logsumexp(z, 1), 0.0)
            del z
            st["g"] = torch.randn(n, generator=g, device="cuda") * (0.3 + 2 * torch.rand(n, generator=g, device="cuda")) / n
            st["dh"] = torch.empty(n, d, device="cuda", dtype=torch.bfloat16)
            st["dw"] = torch.empty(vocab, d, device="cuda", dtype=torch.bfloat16)
        return st
    x, w = _int8_inputs(case, seed)
    st = dict(case=case, x=x, y=torch.empty(case["M"], case["N"], device="cuda", dtype=_dtype(case["out"])))
    if case["kind"] == "int8":
        st["w_q"], st["w_scale"] = _codes(w)
        st["w_image"] = _operand_order(st["w_q"])
    else:
        st["w"] = w.to(_dtype(case["src"]))
        st["w_image"] = torch.empty(case["N"] * case["K"], device="cuda", dtype=torch.int8)
        st["w_scale"] = torch.empty(case["N"], device="cuda")
    return st


# ---- one pass ------------------------------------------------------------------------------------------

def _codes(x):
    """Rows of 8-bit codes and their scales: the largest magnitude of a row is 127, quotients go to the nearest integer, ties to even."""
    scale = (x.abs().amax(1).double() / 127.0).float()   # (a quotient of 32 bits, correctly rounded)
    q = torch.round(x.double() / scale.double()[:, None]).clamp(-127, 127)
    return q.to(torch.int8), scale


def _int8_plain(x, w_q, w_scale, out):
    q, scale = _codes(x)
    return ((q.float() @ w_q.float().T) * scale[:, None] * w_scale[None, :]).to(out)


def _logprob_plain(st):
    z = (st["h"].float() @ st["w"].float().T) * st["it"][:, None]
    top = z.amax(1)
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    has = st["target"] >= 0
    zt = z.gather(1, st["target"].clamp(min=0).long()[:, None])[:, 0]
    return dict(logprob=torch.where(has, zt - lse, 0.0), lse=torch.where(has, lse, 0.0))


def _grad_plain(st):
    h, w = st["h"].float(), st["w"].float()
    z = (h @ w.T) * st["it"][:, None]
    has = st["target"] >= 0
    c = torch.where(has, st["g"] * st["it"], 0.0)
    G = torch.exp(z - st["lse"][:, None]).mul_(-c[:, None])
    G.scatter_add_(1, st["target"].clamp(min=0).long()[:, None], c[:, None])
    return dict(dh=(G @ w).to(torch.bfloat16), dw=(G.T @ h).to(torch.bfloat16))


def _workspace(st, nbytes):
    """The buffer that a program keeps beside its plan."""
    if st.get("workspace") is None:
        st["workspace"] = torch.empty(max(1, nbytes), device="cuda", dtype=torch.uint8)
    return st["workspace"].data_ptr()


def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        if kind == "logprob":
            return _logprob_plain(st)
        if kind == "grad":
            return _grad_plain(st)
        if kind == "int8":
            return dict(y=_int8_plain(st["x"], st["w_q"], st["w_scale"], st["y"].dtype))
        w_q, w_scale = _codes(st["w"])
        return dict(y=_int8_plain(st["x"], w_q, w_scale, st["y"].dtype), w_scale=w_scale)
    import paper_2509_19128_amd as pl
    stream = torch.cuda.current_stream().cuda_stream
    if kind in ("logprob", "grad"):
        n, vocab, d = case["n"], case["vocab"], case["d"]
        p = {k: v.data_ptr() for k, v in st.items() if isinstance(v, torch.Tensor)}
        if kind == "logprob":
            ws = _workspace(st, pl.pl_token_logprob_workspace_bytes(n, vocab, d))
            pl.pl_token_logprob(p["h"], d, p["w"], d, p["target"], p["it"], p["logprob"], p["lse"], n, vocab, d, ws, stream)
            return dict(logprob=st["logprob"], lse=st["lse"])
        ws = _workspace(st, pl.pl_token_logprob_grad_workspace_bytes(n, vocab, d))
        pl.pl_token_logprob_grad(p["h"], d, p["w"], d, p["target"], p["it"], p["lse"], p["g"], p["dh"], p["dw"], n, vocab, d, ws, stream)
        return dict(dh=st["dh"], dw=st["dw"])
    M, N, K = case["M"], case["N"], case["K"]
    dt = lambda t: pl.PL_BF16 if t.dtype == torch.bfloat16 else pl.PL_F32  # noqa: E731
    if kind == "update":
        pl.pl_quantize_int8(st["w"].data_ptr(), dt(st["w"]), K, st["w_image"].data_ptr(), st["w_scale"].data_ptr(), N, K, stream)
    ws = _workspace(st, pl.pl_gemm_int8_workspace_bytes(M, N, K))
    pl.pl_gemm_int8(st["x"].data_ptr(), K, st["w_image"].data_ptr(), st["w_scale"].data_ptr(), st["y"].data_ptr(), dt(st["y"]), M, N, K, ws, stream)
    return dict(y=st["y"], w_scale=st["w_scale"]) if kind == "update" else dict(y=st["y"])


# ---- what a pass cannot do without ---------------------------------------------------------------------

def work(case):
    if case["kind"] in ("logprob", "grad"):
        # (positions without a target have no part in it)
        n, vocab, d = max(1, round(case["n"] * (1 - case["masked"]))), case["vocab"], case["d"]
        operands = 2 * (n + vocab) * d
        if case["kind"] == "logprob":
            return dict(bytes=operands + 16 * n, flops=2 * n * vocab * d)
        # the logits again, then the two products of their gradient
        return dict(bytes=2 * operands + 16 * n, flops=6 * n * vocab * d)
    M, N, K = case["M"], case["N"], case["K"]
    b = 2 * M * K + N * K + 4 * N + (2 if case["out"] == "bf16" else 4) * M * N
    if case["kind"] == "update":
        b += (2 if case["src"] == "bf16" else 4) * N * K + 4 * N   # masters read, codes and scales written (and read above)
    return dict(bytes=b, flops=2 * M * N * K)


# ---- from the definition, in 64 bits -------------------------------------------------------------------

def _quantised64(x):
    """x in 64 bits as its 8-bit codes stand for it; a scale is a 32-bit number."""
    x = x.double()
    s = (x.abs().max(dim=1, keepdim=True).values / 127).float().double()
    return torch.clamp((x / s).round(), min=-127, max=127) * s, s[:, 0]


def exact(case, seed):
    if case["kind"] in ("logprob", "grad"):
        st = prepare(case, seed)
        n, vocab = case["n"], case["vocab"]
        h, w, it, y = st["h"].double(), st["w"].double(), st["it"].double(), st["target"].long()
        rows = torch.nonzero(y >= 0)[:, 0]
        z = torch.mm(h, w.t()).mul_(it[:, None])
        if case["kind"] == "logprob":
            lp, lse = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
            lse[rows] = torch.logsumexp(z[rows], dim=1)
            lp[rows] = z[rows, y[rows]] - lse[rows]
            return dict(logprob=lp, lse=lse)
        # dL/dz of L = sum_t g[t] logprob[t]
        p = z.sub_(st["lse"].double()[:, None]).exp_()
        onehot_minus = p.neg_()
        onehot_minus[rows, y[rows]] += 1.0
        scale = torch.zeros(n, dtype=torch.float64, device="cuda")
        scale[rows] = st["g"].double()[rows] * it[rows]
        dz = onehot_minus.mul_(scale[:, None])
        return dict(dh=torch.mm(dz, w), dw=torch.mm(dz.t(), h))
    st = prepare(case, seed)
    x, _ = _quantised64(st["x"])
    if case["kind"] == "int8":
        return dict(y=torch.mm(x, (st["w_q"].double() * st["w_scale"].double()[:, None]).t()))
    w, s = _quantised64(st["w"])
    # the scales as numbers, before their rounding to 32 bits
    return dict(y=torch.mm(x, w.t()), w_scale=st["w"].double().abs().max(dim=1).values / 127)
