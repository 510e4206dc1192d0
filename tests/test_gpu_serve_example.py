"""The example decoder (examples/serve_requests.py) against its plain forward in fp32, and its ways of serving against each other."""
import importlib.util
import os

import pytest
import torch

from tests.helpers import ensure_built
from tests.helpers import ROOT

pytestmark = pytest.mark.gpu
SIZES = dict(layers=2, hidden=512, heads=8, kv_heads=2, ffn=768, vocab=300, adapters=3, rank=16, pages=40, page=16, positions=128, seed=3)


@pytest.fixture(scope="module")
def S():
    ensure_built()
    spec = importlib.util.spec_from_file_location("serve_requests", os.path.join(ROOT, "examples", "serve_requests.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def weight(e):
    """The matrix that a 4-bit linear stands for."""
    N, K, G = e["N"], e["K"], e["K"] // e["group_size"]
    nibbles = lambda t, n: torch.stack([t.view(N, -1) & 15, t.view(N, -1) >> 4], -1).flatten(1)[:, :n].float()  # noqa: E731
    q, z = nibbles(e["qweight"], K), nibbles(e["zeros"], G)
    return ((q.view(N, G, -1) - z[..., None]) * e["scales"].view(torch.float16).view(N, G, 1).float()).view(N, K)


def plain(m, ids, adapter):
    """Hidden states after the last norm of one request's tokens, in fp32 throughout."""
    norm = lambda h, w: h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-5) * w.float()  # noqa: E731

    def linear(l, x):
        e = l.e
        y = x @ weight(e).t()
        return y if adapter < 0 else y + e["scaling"][adapter] * (x @ e["A"][adapter].float().t()) @ e["B"][adapter].float().t()

    def turned(t):
        half = m.dim // 2
        a, b, c, s = t[..., :half], t[..., half:], m.cos[:len(ids), None], m.sin[:len(ids), None]
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    h = m.embedding[torch.tensor(ids, device="cuda")].float()
    future = torch.ones((len(ids), len(ids)), dtype=torch.bool, device="cuda").triu(1)
    for l in m.layers:
        q, k, v = linear(l["qkv"], norm(h, l["before"])).split((m.heads * m.dim, m.kv_heads * m.dim, m.kv_heads * m.dim), 1)
        q, k, v = (t.unflatten(1, (-1, m.dim)) for t in (q, k, v))
        q, k = turned(q), turned(k).repeat_interleave(m.heads // m.kv_heads, 1)
        v = v.repeat_interleave(m.heads // m.kv_heads, 1)
        o = torch.stack([torch.softmax(((q[:, a] @ k[:, a].t()) * m.dim ** -0.5).masked_fill(future, -torch.inf), 1) @ v[:, a] for a in range(m.heads)], 1)
        h = h + linear(l["out"], o.flatten(1))
        gate, up = linear(l["gate_up"], norm(h, l["after"])).chunk(2, 1)
        h = h + linear(l["down"], gate * torch.sigmoid(gate) * up)
    return norm(h, m.last)


PROMPTS = [[(7 * i + 3 * r) % 300 for i in range(n)] for r, n in enumerate((33, 5, 61))]
ADAPTERS = [2, -1, 0]


@pytest.mark.parametrize("cache", ["bf16", "int8"])
def test_prompts_then_tokens_are_the_plain_forward(S, cache):
    """A packed step of prompts, then one of a few tokens of some requests, then of one token each.  A path from the embedding to the output passes
    about ten roundings to bf16 a layer, each 2^-9 of a row's norm on average (half a step at most, all at once, twice that), and the cache's codes twice
    a layer 1 / 254 of a head's largest value: below 2 * 10 * 2^-8 of a row's norm, 2 * 2 * 2^-6 more with codes."""
    m = S.Decoder(cache=cache, **SIZES)
    table = torch.randperm(40, device="cuda")[:15].view(3, 5).to(torch.int32)
    tol = 20 * 2 ** -8 + (4 * 2 ** -6 if cache == "int8" else 0)
    done = [0, 0, 0]
    for new in ([20, 3, 50], [12, 0, 10], [1, 1, 1]):
        lens = [d + n for d, n in zip(done, new)]
        step = S.Step(m, table, sum(new), max(new), 80)
        step.set(torch.tensor([t for p, d, n in zip(PROMPTS, done, new) for t in p[d:d + n]]), new, lens, ADAPTERS)
        got = step.forward().float().split(new)
        for r in range(3):
            want = plain(m, PROMPTS[r][:lens[r]], ADAPTERS[r])[done[r]:]
            off = (got[r] - want).norm(dim=1) / want.norm(dim=1)
            assert new[r] == 0 or off.max().item() <= tol, (r, off.max().item())
        assert step.errors.item() == 0
        done = lens


@pytest.mark.parametrize("cache", ["bf16", "int8"])
def test_a_captured_step_gives_the_eager_tokens(S, cache):
    m = S.Decoder(cache=cache, **SIZES)
    out, _ = S.serve(m, PROMPTS, ADAPTERS, 8, graph=True)
    again, _ = S.serve(m, PROMPTS, ADAPTERS, 8, graph=False)    # other pages
    assert torch.equal(out, again)


def test_training_step_of_the_last_norm(S):
    m = S.Decoder(**SIZES)
    h = torch.randn((32, 512), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    teacher = (h.float() / h.float().square().mean(1, keepdim=True).sqrt()) @ m.head.float().t()
    losses = [S.train_last_norm(m, h, teacher) for _ in range(6)]
    assert all(b < a for a, b in zip(losses, losses[1:])), losses
