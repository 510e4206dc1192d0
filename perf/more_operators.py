"""The two ends of a policy's decoder, which stay in 16 bits, as cases that can be measured: the lookup of the
tokens' embeddings and its gradient, the product with 16-bit weights that carries bias, activation and residual in
its epilogue (the head, the projector and the vision side's linears) with its gradients, and the choice of the next token.

`run` computes each in its plain form, from elementary torch operations in 32 bits (in 64 where a border decides a
token), or, where `own` is true, by the library's entry points.  `exact` is the same from the definitions in 64 bits.

Sizes are those of the Llama-2-7B backbone (hidden size 4096, 32000 tokens, 11008) and generic ones around them.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

MOST_TABLE = 32000 * 4096
MOST_LOOKED_UP = 24577 * 4096
MOST_MACS = 4096 * 4096 * 11008
MOST_BACK_MACS = 4096 ** 3
MOST_LOGITS = 256 * 32000
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def listed():
    def embed(name, kind, tokens, patches=0, vocab=32000, width=4096, scale=1.0):
        return dict(name=name, kind=kind, tokens=tokens, patches=patches, vocab=vocab, width=width, scale=scale)

    def linear(name, rows, K, N, activation="none", bias=False, residual=False, keep=False, out="bf16"):
        return dict(name=name, kind="linear", rows=rows, K=K, N=N, activation=activation, bias=bias, residual=residual, keep=keep, out=out)

    def back(name, rows, K, N, activation, bias, dy="bf16"):
        return dict(name=name, kind="back", rows=rows, K=K, N=N, activation=activation, bias=bias, dy=dy)

    def sample(name, rows, vocab, dtype):
        return dict(name=name, kind="sample", rows=rows, vocab=vocab, dtype=dtype, mix=7)

    return [
        # a decode step of 16 requests.  The smallest call
        embed("embed_decode", "embed", 16),
        # packed prompts, scaled; a quarter of the rows hold image patches, which the projector writes and the lookup leaves alone
        embed("embed_prompts", "embed", 8229, patches=2048, scale=8.0),
        # training: a short batch; and a long one, in which the commonest token comes about 1600 times
        embed("embed_gradient", "embed_back", 2312),
        embed("embed_gradient_long", "embed_back", 24577, patches=4096, scale=64.0),
        # the head of a decode step of 16 requests: real-valued logits
        linear("head_decode", 16, 4096, 32000, out="fp32"),
        # the first linear of a vision block, 8 frames of 257 patches; z is kept for the backward pass
        linear("patches_gelu", 2056, 1024, 4096, activation="gelu", bias=True, keep=True),
        # a wide linear of a long prompt with everything in its epilogue
        linear("long_silu_residual", 4096, 4096, 11008, activation="silu", bias=True, residual=True),
        # training: the projector's second linear on one prompt, an odd number of rows
        back("gradient_gelu", 289, 4096, 4096, "gelu", True),
        # training: a long batch
        back("gradient_long", 4096, 4096, 4096, "gelu_tanh", True),
        # the next token of one request
        sample("sample_one", 1, 32000, "fp32"),
        # ... of many, each with choices of its own
        sample("sample_many", 256, 32000, "bf16"),
        # ... from a large vocabulary
        sample("sample_wide", 48, 131072, "fp32"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_embed(rng, kind):
    width = rng.choice((1024, 2048, 4096, 5120, 8 * _log(rng, 8, 1024), 8 * (2 * _log(rng, 4, 500) + 1)))
    vocab = _log(rng, 64, min(65536, MOST_TABLE // width))
    tokens = _log(rng, 1, min(24577, MOST_LOOKED_UP // width))
    return dict(kind=kind, tokens=tokens, patches=rng.choice((0, 0, tokens // 3)), vocab=vocab, width=width, scale=rng.choice((1.0, 1.0, float(math.isqrt(width)))))


def _sizes(rng, most):
    while True:
        rows = _log(rng, 1, 4096)
        K = rng.choice((1024, 4096, 8 * _log(rng, 4, 1376), 8 * (2 * _log(rng, 2, 600) + 1)))
        N = rng.choice((1024, 4096, 11008, 32000, 2 * _log(rng, 8, 8000) + 1, 8 * _log(rng, 2, 1400)))
        if rows * K * N <= most and N * K <= MOST_TABLE:
            return dict(rows=rows, K=K, N=N)


def draw(rng):
    kind = rng.choice(("embed", "embed_back", "linear", "linear", "back", "back", "sample", "sample"))
    if kind in ("embed", "embed_back"):
        return _draw_embed(rng, kind)
    if kind == "sample":
        vocab = _log(rng, 200, 131072)
        return dict(kind=kind, rows=_log(rng, 1, min(256, MOST_LOGITS // vocab)), vocab=vocab, dtype=rng.choice(("bf16", "fp32")), mix=rng.randint(1, 10 ** 6))
    activation = rng.choice(ACTIVATIONS)
    if kind == "back":
        return dict(kind=kind, **_sizes(rng, MOST_BACK_MACS), activation=activation, bias=rng.random() < 0.6, dy=rng.choice(("bf16", "bf16", "fp32")))
    return dict(kind=kind, **_sizes(rng, MOST_MACS), activation=activation, bias=rng.random() < 0.6, residual=rng.random() < 0.4,
                keep=rng.random() < 0.4, out=rng.choice(("bf16", "bf16", "fp32")))


# ------------------------------------------------------------------------------------- inputs --

def _rng(seed, stream):
    return torch.Generator(device="cuda").manual_seed(1013 * int(seed) + stream)


def _normal(shape, seed, stream, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=_rng(seed, stream), device="cuda") * std).to(dtype)


def _hidden(rows, width, seed, stream):
    """Hidden states: a few columns are ten times as large."""
    t = torch.randn((rows, width), generator=_rng(seed, stream), device="cuda")
    t[:, torch.randperm(width, generator=_rng(seed, stream + 1), device="cuda")[: math.ceil(0.005 * width)]] *= 10
    return t.to(torch.bfloat16)


def _prepare_embed(case, seed):
    T, V, K = case["tokens"], case["vocab"], case["width"]
    # how often a token comes falls with its rank as 1 / rank; ranks are spread over the vocabulary
    rank = torch.rand((T,), generator=_rng(seed, 1), device="cuda", dtype=torch.float64).mul_(math.log(V + 1)).exp_().long().sub_(1).clamp_(0, V - 1)
    ids = torch.randperm(V, generator=_rng(seed, 2), device="cuda")[rank].to(torch.int32)
    for start in range(0, case["patches"], 256):    # frames of up to 256 patches, evenly spread
        n = min(256, case["patches"] - start)
        at = start * T // max(1, case["patches"])
        ids[at:at + n] = -1
    st = dict(ids=ids)
    if case["kind"] == "embed":
        st.update(table=_normal((V, K), seed, 3), h=_hidden(T, K, seed, 4))    # (h holds the patches' rows)
    else:
        st["dh"] = _normal((T, K), seed, 5)
    return st


def _prepare_linear(case, seed):
    M, N, K = case["rows"], case["N"], case["K"]
    st = dict(x=_hidden(M, K, seed, 1), weight=_normal((N, K), seed, 3, K ** -0.5), bias=_normal((N,), seed, 4, 0.2) if case["bias"] else None)
    if case["kind"] == "linear":
        st["residual"] = _hidden(M, N, seed, 5) if case["residual"] else None
    else:
        st["z"] = _normal((M, N), seed, 7) if case["activation"] != "none" else None
        st["dy"] = _normal((M, N), seed, 8, dtype=torch.bfloat16 if case["dy"] == "bf16" else torch.float32)
    return st


def _prepare_sample(case, seed):
    R, V = case["rows"], case["vocab"]
    rng = random.Random(case["mix"] + 1000003 * int(seed))
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    width = torch.tensor([1.5 + 2.0 * rng.random() for _ in range(R)], device="cuda")[:, None]
    logits = torch.randn((R, V), generator=_rng(seed, 1), device="cuda") * width
    some = torch.randint(0, V, (R, 12), generator=_rng(seed, 2), device="cuda")    # what the context makes likely
    logits.scatter_add_(1, some, 4 + 6 * torch.rand((R, 12), generator=_rng(seed, 3), device="cuda"))
    for r in range(1, R):
        if rng.random() < 0.15:    # only some tokens are allowed: the policy's actions
            first = rng.randint(0, V // 2)
            logits[r, :first] = -math.inf
            logits[r, first + max(1, V // 8):] = -math.inf
    # a request's choices, the first one's the commonest: (temperature, top-k, top-p, min-p)
    choices = [(0.8, 0, 0.95, 0.0)] + [(rng.choice((0.0, 0.6, 0.8, 1.0, 1.0, 1.3)), rng.choice((0, 0, 0, 1, 20, 50, 400)), rng.choice((1.0, 1.0, 0.5, 0.9, 0.95)),
                                        rng.choice((0.0, 0.0, 0.02, 0.1))) for _ in range(R - 1)]
    t, k, p, m = zip(*choices)
    column = lambda v, dtype=torch.float32: torch.tensor(v, dtype=dtype, device="cuda")  # noqa: E731
    return dict(logits=logits.to(dtype), u=torch.rand((R,), generator=_rng(seed, 4), device="cuda"), temperature=column(t),
                top_k=column(k, torch.int32), top_p=column(p), min_p=column(m))


def prepare(case, seed):
    make = {"embed": _prepare_embed, "embed_back": _prepare_embed, "linear": _prepare_linear, "back": _prepare_linear, "sample": _prepare_sample}
    return dict(make[case["kind"]](case, seed), case=case)


# -------------------------------------------------------------------------------- plain forms --

def _plain_embed(st):
    ids = st["ids"].long()
    rows = (st["table"][ids.clamp(min=0)].float() * st["case"]["scale"]).to(torch.bfloat16)
    return torch.where((ids < 0)[:, None], st["h"], rows)


def _plain_embed_back(st):
    c, ids = st["case"], st["ids"].long()
    held = ids >= 0
    out = torch.zeros((c["vocab"], c["width"]), device="cuda")
    return out.index_add_(0, ids.clamp(min=0), st["dh"].float() * held[:, None]).mul_(c["scale"])


def _activated(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if name == "silu" else z


def _slope(name, z):
    if name == "relu":
        return (z > 0).float()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


def _plain_linear(st):
    c = st["case"]
    z = st["x"].float() @ st["weight"].float().t()
    if st["bias"] is not None:
        z = z + st["bias"].float()
    y = _activated(c["activation"], z)
    if st["residual"] is not None:
        y = y + st["residual"].float()
    out = dict(y=y if c["out"] == "fp32" else y.to(torch.bfloat16))
    return dict(out, z=z.to(torch.bfloat16)) if c["keep"] else out


def _plain_back(st):
    c = st["case"]
    dz = st["dy"].float()
    if c["activation"] != "none":
        dz = dz * _slope(c["activation"], st["z"].float())
    out = dict(dx=(dz @ st["weight"].float()).to(torch.bfloat16), dweight=(dz.t() @ st["x"].float()).to(torch.bfloat16))
    return dict(out, dbias=dz.sum(0)) if c["bias"] else out


def _plain_sample(st):
    x, V = st["logits"].double(), st["case"]["vocab"]
    at = torch.arange(V, device="cuda")
    most = x.amax(1, keepdim=True)
    first = torch.where(x == most, at, V).amin(1)
    t = st["temperature"].double()[:, None]
    down, order = ((x - most) / torch.where(t > 0, t, 1.0)).sort(dim=1, descending=True, stable=True)    # ties: the lowest index first
    k = st["top_k"].long()[:, None]
    w = torch.where(at < torch.where(k > 0, k, V), down.exp(), 0.0)
    upto = w.cumsum(1)
    before = torch.cat((torch.zeros_like(upto[:, :1]), upto[:, :-1]), 1)
    kept = (before < st["top_p"].double()[:, None] * upto[:, -1:]) & (w >= st["min_p"].double()[:, None])
    kept[:, 0] = True
    w = torch.zeros_like(w).scatter_(1, order, torch.where(kept, w, 0.0))
    upto = w.cumsum(1)
    total = upto[:, -1:]
    token = (upto <= st["u"].double()[:, None] * total).sum(1)
    logprob = (w.gather(1, token[:, None]) / total).log()[:, 0]
    greedy = st["temperature"] == 0
    return dict(token=torch.where(greedy, first, token).to(torch.int32), logprob=torch.where(greedy, 0.0, logprob).float())


# -------------------------------------------------------------------------- the library's calls --

def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def _own_embed(st):
    from paper_2412_01034_amd import binding as B
    B.qail_embed(st["table"], st["ids"], st["h"], scale=st["case"]["scale"])
    return st["h"]


def _own_embed_back(st):
    from paper_2412_01034_amd import binding as B
    c = st["case"]
    if "out" not in st:
        st["out"] = torch.empty((c["vocab"], c["width"]), device="cuda")
        st["workspace"] = _bytes(B.qail_embed_backward_workspace(c["vocab"], c["width"], c["tokens"]))
    B.qail_embed_backward(st["ids"], st["dh"], st["out"], st["workspace"], scale=c["scale"])
    return st["out"]


def _own_linear(st):
    from paper_2412_01034_amd import binding as B
    c = st["case"]
    if "handle" not in st:
        st["handle"] = B.make_w16a16(st["weight"], st["bias"], c["activation"])
        st["out"] = dict(y=torch.empty((c["rows"], c["N"]), device="cuda", dtype=torch.float32 if c["out"] == "fp32" else torch.bfloat16))
        if c["keep"]:
            st["out"]["z"] = torch.empty((c["rows"], c["N"]), device="cuda", dtype=torch.bfloat16)
        st["workspace"] = _bytes(B.qail_w16a16_workspace(st["handle"], c["rows"]))
    B.qail_w16a16_linear(st["handle"], st["x"], st["out"]["y"], st["workspace"], residual=st["residual"], z=st["out"].get("z"))
    return st["out"]


def _own_back(st):
    from paper_2412_01034_amd import binding as B
    c = st["case"]
    if "handle" not in st:
        st["handle"] = B.make_w16a16(st["weight"], st["bias"], c["activation"])
        st["out"] = dict(dx=torch.empty_like(st["x"]), dweight=torch.empty_like(st["weight"]))
        if c["bias"]:
            st["out"]["dbias"] = torch.empty((c["N"],), device="cuda")
        st["workspace"] = _bytes(B.qail_w16a16_backward_workspace(st["handle"], c["rows"]))
    out = st["out"]
    B.qail_w16a16_backward(st["handle"], st["x"], st["dy"], st["workspace"], z=st["z"], dx=out["dx"], dweight=out["dweight"], dbias=out.get("dbias"))
    return out


def _own_sample(st):
    from paper_2412_01034_amd import binding as B
    if "out" not in st:
        rows = st["case"]["rows"]
        st["out"] = dict(token=torch.empty((rows,), dtype=torch.int32, device="cuda"), logprob=torch.empty((rows,), device="cuda"))
    B.qail_sample(st["logits"], st["u"], st["out"]["token"], logprob=st["out"]["logprob"], temperature=st["temperature"], top_k=st["top_k"],
                  top_p=st["top_p"], min_p=st["min_p"])
    return st["out"]


def run(st):
    plain = {"embed": _plain_embed, "embed_back": _plain_embed_back, "linear": _plain_linear, "back": _plain_back, "sample": _plain_sample}
    mine = {"embed": _own_embed, "embed_back": _own_embed_back, "linear": _own_linear, "back": _own_back, "sample": _own_sample}
    return (mine if own else plain)[st["case"]["kind"]](st)


# --------------------------------------------------------------------------------------- work --

def work(case):
    kind = case["kind"]
    if kind in ("embed", "embed_back"):
        T, V, K = case["tokens"] - case["patches"], case["vocab"], case["width"]
        if kind == "embed_back":
            return dict(bytes=4 * case["tokens"] + 2 * T * K + 4 * V * K, flops=T * K)
        distinct = sum(1 - (1 - math.log((i + 1) / i) / math.log(V + 1)) ** T for i in range(1, V + 1))    # rows read, on average
        return dict(bytes=int(4 * case["tokens"] + 2 * distinct * K + 2 * T * K), flops=T * K)
    if kind == "sample":
        n = case["rows"] * case["vocab"]
        return dict(bytes=n * (2 if case["dtype"] == "bf16" else 4) + 28 * case["rows"], flops=20 * n)
    M, N, K = case["rows"], case["N"], case["K"]
    if kind == "back":
        byte = 2 * M * K + 2 * N * K + M * N * (2 if case["dy"] == "bf16" else 4) + (2 * M * N if case["activation"] != "none" else 0)
        return dict(bytes=byte + 2 * M * K + 2 * N * K + (4 * N if case["bias"] else 0), flops=4 * M * N * K)
    byte = 2 * M * K + 2 * N * K + M * N * (4 if case["out"] == "fp32" else 2) + (2 * N if case["bias"] else 0)
    return dict(bytes=byte + 2 * M * N * (int(case["residual"]) + int(case["keep"])), flops=2 * M * N * K)


# -------------------------------------------------------------------------------------- exact --

def _exact_embed(st):
    out = st["h"].double()
    for t, i in enumerate(st["ids"].tolist()):
        if i >= 0:
            out[t] = st["table"][i].double() * st["case"]["scale"]
    return out


def _exact_embed_back(st):
    c = st["case"]
    out = torch.zeros((c["vocab"], c["width"]), dtype=torch.float64, device="cuda")
    where = {}
    for t, i in enumerate(st["ids"].tolist()):
        where.setdefault(i, []).append(t)
    for i, rows in where.items():
        if i >= 0:
            out[i] = st["dh"][torch.tensor(rows, device="cuda")].double().sum(0) * c["scale"]
    return out


def _exact_function(name, z):
    """act(z) and its derivative."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return torch.maximum(z, torch.zeros_like(z)), torch.where(z > 0, 1.0, 0.0).double()
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s + z * s * (1 - s)
    if name == "gelu":
        share = 0.5 * torch.erfc(-z / math.sqrt(2))    # of the normal distribution below z
        return z * share, share + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    a = math.sqrt(2 / math.pi)
    share = 1 / (1 + torch.exp(-2 * a * (z + 0.044715 * z * z * z)))    # (1 + tanh(v)) / 2
    return z * share, share + 2 * a * z * share * (1 - share) * (1 + 0.134145 * z * z)


def _exact_linear(st):
    c = st["case"]
    z = torch.matmul(st["x"].double(), st["weight"].double().t().contiguous())
    if st["bias"] is not None:
        z += st["bias"].double()
    y = _exact_function(c["activation"], z)[0]
    if st["residual"] is not None:
        y = y + st["residual"].double()
    return dict(y=y, z=z) if c["keep"] else dict(y=y)


def _exact_back(st):
    c = st["case"]
    dz = st["dy"].double()
    if c["activation"] != "none":
        dz = dz * _exact_function(c["activation"], st["z"].double())[1]
    out = dict(dx=torch.matmul(dz, st["weight"].double()), dweight=torch.matmul(dz.t().contiguous(), st["x"].double()))
    return dict(out, dbias=torch.sum(dz, 0)) if c["bias"] else out


def _exact_sample(st):
    token, logprob = [], []
    t, k, p, m, u = (st[n].double().cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p", "u"))
    for r, x in enumerate(st["logits"].double().cpu().numpy()):
        order = np.argsort(-x, kind="stable")
        if t[r] == 0:
            token.append(int(order[0]))
            logprob.append(0.0)
            continue
        if k[r] > 0:
            order = order[:int(k[r])]
        w = np.exp((x[order] - x[order[0]]) / t[r])
        if p[r] < 1:
            n = 1 + int(np.searchsorted(np.cumsum(w), p[r] * np.sum(w), side="left"))    # the first n reach the share
            order, w = order[:n], w[:n]
        n = max(1, int(np.sum(w >= m[r])))
        order, w = order[:n], w[:n]
        by = np.argsort(order)
        upto = np.cumsum(w[by])
        i = int(np.searchsorted(upto, u[r] * upto[-1], side="right"))
        token.append(int(order[by[i]]))
        logprob.append(math.log(w[by[i]] / upto[-1]))
    return dict(token=torch.tensor(token, dtype=torch.int32, device="cuda"), logprob=torch.tensor(logprob, dtype=torch.float64, device="cuda"))


def exact(case, seed):
    how = {"embed": _exact_embed, "embed_back": _exact_embed_back, "linear": _exact_linear, "back": _exact_back, "sample": _exact_sample}
    return how[case["kind"]](prepare(case, seed))
