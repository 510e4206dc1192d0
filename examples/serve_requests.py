#!/usr/bin/env python3
"""Several requests served by one decoder of 4-bit linears: prompts of different lengths in one packed step, then a token each in a
captured graph, each request with an adapter of its own (or none) and its keys and values in pages, greedy or drawn (`--temperature`); then training steps of
the last norm against the logits of a teacher, and of the embeddings under it (`--train`).  Random weights; sizes as the options say.

    python examples/serve_requests.py [--layers 2 --hidden 1024 --heads 8 --kv-heads 2 --ffn 2816 --tokens 16 --cache int8 --temperature 0.8 --top-p 0.95]

Where each of the library's calls stands around the layers and in one:

    qail_embed -> layers -> qail_rmsnorm -> qail_w16a16_linear (the head) -> qail_sample

    qail_rmsnorm -> linears (qail_w4a16_linear_adapters_batch) -> qail_kv_append -> qail_paged_attention -> linear
    qail_rmsnorm -> linear -> silu(gate) * up -> linear
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2412_01034_amd import binding as B  # noqa: E402

BF16 = torch.bfloat16
GROUP = 128
EPS = 1e-5


class Linear:
    """A 4-bit linear, quantised by the library, and its stack of adapters."""

    def __init__(self, N, K, adapters, rank, generator):
        normal = lambda *shape: torch.randn(shape, generator=generator, device="cuda")  # noqa: E731
        q, s, z = B.qail_packed_sizes(N, K, GROUP, B.QAIL_W4_ASYM_GROUP)
        new = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.e = dict(N=N, K=K, group_size=GROUP, qweight=new(q), scales=new(s), zeros=new(z), A=(normal(adapters, rank, K) * K ** -0.5).to(BF16),
                      B=(normal(adapters, N, rank) * 0.3 * rank ** -0.5).to(BF16), scaling=torch.full((adapters,), 1.0, device="cuda"))
        B.qail_quantize_weights(normal(N, K) * K ** -0.5, GROUP, B.QAIL_W4_ASYM_GROUP, self.e["qweight"], self.e["scales"], self.e["zeros"])


class Decoder:
    """The weights, and a cache of keys and values in pages for each layer."""

    def __init__(self, layers=2, hidden=1024, heads=8, kv_heads=2, ffn=2816, vocab=2048, adapters=3, rank=16, pages=64, page=16, positions=1024,
                 cache="bf16", seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.hidden, self.heads, self.kv_heads, self.dim, self.page, self.ffn = hidden, heads, kv_heads, hidden // heads, page, ffn
        normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
        self.embedding, self.head = normal(vocab, hidden).to(BF16), (normal(vocab, hidden) * hidden ** -0.5).to(BF16)
        norm = lambda: (1 + 0.1 * normal(hidden)).to(BF16)  # noqa: E731
        wide = (heads + 2 * kv_heads) * self.dim
        self.layers = [dict(before=norm(), after=norm(), qkv=Linear(wide, hidden, adapters, rank, g), out=Linear(hidden, hidden, adapters, rank, g),
                            gate_up=Linear(2 * ffn, hidden, adapters, rank, g), down=Linear(hidden, ffn, adapters, rank, g)) for _ in range(layers)]
        self.last = norm()
        self.head16 = B.make_w16a16(self.head)
        for layer in self.layers:
            shape = (pages, kv_heads, page, self.dim)
            layer["kv"] = [torch.zeros(shape, dtype=torch.int8 if cache == "int8" else BF16, device="cuda") for _ in range(2)]
            if cache == "int8":
                layer["kv"] += [torch.zeros(shape[:3], device="cuda") for _ in range(2)]
            layer["cache"] = B.make_kv_cache(*layer["kv"])
        angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(self.dim // 2, device="cuda", dtype=torch.float64) * 2 / self.dim)
        self.cos, self.sin = angle.cos().float(), angle.sin().float()


class Step:
    """The buffers of steps of `tokens` tokens of `requests` requests, and one pass through the decoder with them.  What the requests are is
    in device memory (q_start, kv_len, the page table, the tokens and their adapters): one step, captured, serves any of them."""

    def __init__(self, model, table, tokens, max_new, max_len):
        m, new = model, lambda *shape: torch.empty(shape, dtype=BF16, device="cuda")
        self.model, self.tokens = m, tokens
        whole = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
        R = table.shape[0]
        self.ids, self.q_start, self.kv_len, self.row_adapter = whole(tokens), whole(R + 1), whole(R), whole(tokens)
        self.table, self.errors = table, whole(1)
        self.requests = B.make_requests(table, self.q_start, self.kv_len, tokens=tokens, max_new=max_new, max_len=max_len)
        self.h, self.y, self.qkv = new(tokens, m.hidden), new(tokens, m.hidden), new(tokens, (m.heads + 2 * m.kv_heads) * m.dim)
        a, b = m.heads * m.dim, m.kv_heads * m.dim
        self.q, self.k, self.v = (t.unflatten(1, (-1, m.dim)) for t in self.qkv.split((a, b, b), dim=1))
        self.turned, self.attended = new(tokens, m.heads, m.dim), new(tokens, m.heads, m.dim)
        self.gate_up, self.act = new(tokens, 2 * m.ffn), new(tokens, m.ffn)
        need = 0
        self.calls = []
        for layer in m.layers:
            made = {}
            for name, x, y in (("qkv", self.y, self.qkv), ("out", self.attended, self.y), ("gate_up", self.y, self.gate_up), ("down", self.act, self.y)):
                e = dict(layer[name].e, x=x, y=y)
                made[name] = B.make_w4a16_items([e], tokens), B.make_adapters([e])
                need = max(need, B.qail_w4a16_adapters_workspace(*made[name], 1, tokens))
            need = max(need, B.qail_paged_attention_workspace(layer["cache"], self.requests, m.heads))
            self.calls.append(made)
        self.rows, self.logit = new(R, m.hidden), torch.empty((R, m.head.shape[0]), device="cuda")
        self.token, self.u, self.choice = whole(R), torch.zeros(R, device="cuda"), {"temperature": torch.zeros(R, device="cuda")}    # greedy
        need = max(need, B.qail_w16a16_workspace(m.head16, R))
        self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")

    def set(self, ids, new, lens, adapters):
        """The requests of the next pass: their packed tokens, how many each has, its length with them and its adapter (-1: none)."""
        of = torch.tensor(adapters).repeat_interleave(torch.tensor(new))
        self.ids.copy_(ids)
        self.q_start.copy_(torch.tensor([0] + new).cumsum(0))
        self.kv_len.copy_(torch.tensor(lens))
        self.row_adapter.copy_(of)

    def linear(self, call):
        B.qail_w4a16_linear_adapters_batch(*call, self.row_adapter, 1, self.tokens, self.workspace)

    def forward(self):
        """Hidden states after the last norm, [tokens, hidden] (the step's own buffer)."""
        m = self.model
        B.qail_embed(m.embedding, self.ids, self.h, errors=self.errors)
        for i, (layer, call) in enumerate(zip(m.layers, self.calls)):
            if i == 0:
                B.qail_rmsnorm(self.h, layer["before"], EPS, y=self.y)
            else:    # y holds what the layer before has added
                B.qail_rmsnorm(self.y, layer["before"], EPS, residual=self.h, residual_out=self.h, y=self.y)
            self.linear(call["qkv"])
            B.qail_kv_append(layer["cache"], self.requests, self.k, self.v, q=self.q, q_out=self.turned, cos=m.cos, sin=m.sin, errors=self.errors)
            B.qail_paged_attention(layer["cache"], self.requests, self.turned, self.attended, m.dim ** -0.5, self.workspace, errors=self.errors)
            self.linear(call["out"])
            B.qail_rmsnorm(self.y, layer["after"], EPS, residual=self.h, residual_out=self.h, y=self.y)
            self.linear(call["gate_up"])
            gate, up = self.gate_up.chunk(2, 1)
            torch.mul(torch.nn.functional.silu(gate), up, out=self.act)
            self.linear(call["down"])
        B.qail_rmsnorm(self.y, m.last, EPS, residual=self.h, residual_out=self.h, y=self.y)
        return self.y

    def logits(self):
        """Of each request's last token, [requests, vocab] (the step's own buffer)."""
        torch.index_select(self.y, 0, self.q_start[1:] - 1, out=self.rows)
        B.qail_w16a16_linear(self.model.head16, self.rows, self.logit, self.workspace)
        return self.logit

    def next(self):
        """The next token of each request, drawn at the random numbers `u` as `choice` says."""
        B.qail_sample(self.logits(), self.u, self.token, errors=self.errors, **self.choice)
        return self.token


def serve(model, prompts, adapters, tokens, graph=True, choice=None, seed=0):
    """`tokens` tokens for each prompt (a list of token numbers): [requests, tokens], and seconds per decode step.  Greedy, or drawn as `choice` says (temperature, top_k,
    top_p, min_p: a number for all requests)."""
    R, page = len(prompts), model.page
    lens = [len(p) for p in prompts]
    most = max(lens) + tokens
    per = -(-most // page)
    free = model.layers[0]["kv"][0].shape[0]
    if R * per > free:
        raise ValueError("%d pages are needed, %d are there" % (R * per, free))
    table = torch.randperm(free, device="cuda")[:R * per].view(R, per).to(torch.int32)    # the cache's pages in any order
    first = Step(model, table, sum(lens), max(lens), most)
    first.set(torch.tensor([t for p in prompts for t in p]), lens, lens, adapters)
    step = Step(model, table, R, 1, most)
    if choice is not None:
        first.choice = step.choice = {k: torch.full((R,), v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in choice.items()}
    random = torch.Generator(device="cuda").manual_seed(seed)
    first.u.uniform_(generator=random)
    first.forward()
    out = [first.next().clone()]
    step.set(out[0], [1] * R, [n + 1 for n in lens], adapters)

    def run():
        step.forward()
        step.next()

    if graph:
        run()    # (the token that is appended is appended again by the first replay)
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            run()
        run = captured.replay
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(tokens - 1):
        step.u.uniform_(generator=random)
        run()
        out.append(step.token.clone())
        step.ids.copy_(step.token)
        step.kv_len += 1
    torch.cuda.synchronize()
    seconds = (time.perf_counter() - t0) / max(1, tokens - 1)
    if first.errors.item() or step.errors.item():
        raise RuntimeError("bad requests")
    return torch.stack(out, 1), seconds


def loss_of(model, h, teacher):
    """The distance of the logits of hidden states `h` from a teacher's, and its gradients at h (before the last norm) and at the norm's weight."""
    rows, hidden = h.shape
    y, logits = torch.empty_like(h), torch.empty((rows, model.head.shape[0]), device="cuda")
    need = max(B.qail_w16a16_workspace(model.head16, rows), B.qail_w16a16_backward_workspace(model.head16, rows), B.qail_rmsnorm_backward_workspace(rows, hidden), rows * 4)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    B.qail_rmsnorm(h, model.last, EPS, y=y)
    B.qail_w16a16_linear(model.head16, y, logits, ws)
    loss, grad = torch.empty(1, device="cuda"), torch.empty_like(logits)
    B.qail_qbc_loss(logits, teacher, loss, grad, ws)
    dy, dh, dweight = torch.empty_like(h), torch.empty_like(h), torch.empty(hidden, device="cuda")
    B.qail_w16a16_backward(model.head16, None, grad, ws, dx=dy)
    B.qail_rmsnorm_backward(h, model.last, EPS, dy, dh, dweight, ws)
    return loss, dh, dweight


def train_last_norm(model, h, teacher, rate=0.5):
    """One step of the last norm's weight towards a teacher's logits of the hidden states `h`; the loss before it."""
    loss, _, dweight = loss_of(model, h, teacher)
    model.last = (model.last.float() - rate * dweight).to(BF16)
    return loss.item()


def embedding_gradient(model, ids, teacher):
    """The loss of the embeddings of `ids` themselves as hidden states, and its gradient at the table: fp32 [vocab, hidden]."""
    vocab, hidden = model.embedding.shape
    h, dtable = torch.empty((ids.numel(), hidden), dtype=BF16, device="cuda"), torch.empty((vocab, hidden), device="cuda")
    B.qail_embed(model.embedding, ids, h)
    loss, dh, _ = loss_of(model, h, teacher)
    ws = torch.empty(B.qail_embed_backward_workspace(vocab, hidden, ids.numel()), dtype=torch.uint8, device="cuda")
    B.qail_embed_backward(ids, dh, dtable, ws)
    return loss.item(), dtable


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("layers", 2), ("hidden", 1024), ("heads", 8), ("kv-heads", 2), ("ffn", 2816), ("tokens", 16), ("requests", 4)):
        p.add_argument("--" + name, type=int, default=default)
    p.add_argument("--cache", choices=("bf16", "int8"), default="bf16")
    p.add_argument("--temperature", type=float, default=0.0, help="0: greedy")
    p.add_argument("--top-k", type=int, default=0)
    p.add_argument("--top-p", type=float, default=1.0)
    p.add_argument("--min-p", type=float, default=0.0)
    p.add_argument("--train", action="store_true")
    a = p.parse_args()
    model = Decoder(a.layers, a.hidden, a.heads, a.kv_heads, a.ffn, cache=a.cache, pages=a.requests * 32)
    prompts = [torch.randint(0, 2048, (20 + 37 * i % 200,), generator=torch.Generator().manual_seed(i)).tolist() for i in range(a.requests)]
    adapters = [i % 4 - 1 for i in range(a.requests)]
    out, seconds = serve(model, prompts, adapters, a.tokens, choice=dict(temperature=a.temperature, top_k=a.top_k, top_p=a.top_p, min_p=a.min_p))
    for r, row in enumerate(out.tolist()):
        print("request %d: %d tokens, adapter %d ->" % (r, len(prompts[r]), adapters[r]), *row)
    print("a decode step of %d requests: %.0f us" % (a.requests, seconds * 1e6))
    if a.train:
        h = torch.randn((64, a.hidden), device="cuda").to(BF16)
        teacher = (h.float() / h.float().square().mean(1, keepdim=True).sqrt()) @ model.head.float().t()
        print("loss of the last norm:", *("%.4f" % train_last_norm(model, h, teacher) for _ in range(8)))
        loss, dtable = embedding_gradient(model, torch.arange(64, dtype=torch.int32, device="cuda") % 10, teacher)
        print("loss of ten tokens' embeddings: %.4f, rows of the table with a gradient: %d" % (loss, dtable.abs().amax(1).count_nonzero().item()))


if __name__ == "__main__":
    main()
