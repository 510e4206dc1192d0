"""The policy's ends used together: tokens to logits to tokens in a captured graph, on other streams, with image patches between the tokens, and the way back through
the head, the norm and the embeddings."""
import importlib.util
import math
import os

import pytest
import torch

from tests.helpers import ROOT, ensure_built

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
EPS = 1e-5


@pytest.fixture(scope="module")
def B():
    return ensure_built()


@pytest.fixture(scope="module")
def S():
    ensure_built()
    spec = importlib.util.spec_from_file_location("serve_requests", os.path.join(ROOT, "examples", "serve_requests.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


SIZES = dict(layers=2, hidden=512, heads=8, kv_heads=2, ffn=768, vocab=300, adapters=3, rank=16, pages=40, page=16, positions=128, seed=3)
PROMPTS = [[(7 * i + 3 * r) % 300 for i in range(n)] for r, n in enumerate((33, 5, 61))]


def normal(shape, seed, std=1.0, dtype=BF16):
    return (torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * std).to(dtype)


def space(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")


class Model:
    """Embeddings, a projector of image patches into them, a norm, a head: everything of a policy but its layers."""

    def __init__(self, B, vocab, hidden, patch, tokens, patches):
        self.B, self.patches = B, patches
        self.table, self.head = normal((vocab, hidden), 1), normal((vocab, hidden), 2, hidden ** -0.5)
        self.projector, self.bias, self.norm = normal((hidden, patch), 3, patch ** -0.5), normal((hidden,), 4), (1 + normal((hidden,), 5, 0.1, torch.float32)).to(BF16)
        self.features = normal((patches, patch), 6)
        self.p, self.d = B.make_w16a16(self.projector, self.bias, "gelu"), B.make_w16a16(self.head)
        self.ids = torch.zeros(tokens, dtype=torch.int32, device="cuda")
        self.h, self.y = torch.empty((tokens, hidden), dtype=BF16, device="cuda"), torch.empty((tokens, hidden), dtype=BF16, device="cuda")
        self.logits, self.u = torch.empty((tokens, vocab), device="cuda"), torch.zeros(tokens, device="cuda")
        self.token, self.logprob = torch.empty(tokens, dtype=torch.int32, device="cuda"), torch.empty(tokens, device="cuda")
        self.ws = space(max(B.qail_w16a16_workspace(self.p, max(1, patches)), B.qail_w16a16_workspace(self.d, tokens)))

    def run(self, **choice):
        B = self.B
        if self.patches:
            B.qail_w16a16_linear(self.p, self.features, self.h[:self.patches], self.ws)     # the patches' rows, which the lookup leaves alone
        B.qail_embed(self.table, self.ids, self.h, scale=2.0)
        B.qail_rmsnorm(self.h, self.norm, EPS, y=self.y)
        B.qail_w16a16_linear(self.d, self.y, self.logits, self.ws)
        B.qail_sample(self.logits, self.u, self.token, logprob=self.logprob, **choice)
        return self.token

    def set(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.ids.copy_(torch.randint(0, self.table.shape[0], self.ids.shape, generator=g, device="cuda"))
        self.ids[:self.patches] = -1
        self.u.uniform_(generator=g)


def choices(R, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    pick = lambda *v, dtype=torch.float32: torch.tensor(v, dtype=dtype, device="cuda")[torch.randint(0, len(v), (R,), generator=g, device="cuda")]  # noqa: E731
    return dict(temperature=pick(0.0, 0.7, 1.0), top_k=pick(0, 5, 40, dtype=torch.int32), top_p=pick(1.0, 0.9), min_p=pick(0.0, 0.05))


@pytest.mark.parametrize("vocab, hidden, patch, tokens, patches", [(1000, 512, 136, 70, 33), (257, 72, 40, 5, 2), (2003, 1024, 64, 300, 0)])
def test_tokens_to_tokens(B, vocab, hidden, patch, tokens, patches):
    """Against the same in 64 bits from the rows that the calls round to bf16: h is one rounding of 2^-8 off, y by two more (h's, and its own, of the
    row's norm: below 3 * 2^-8 with the weight's 1.5), logits by that of |y| |head| at most; the token is the one that the logits say."""
    m = Model(B, vocab, hidden, patch, tokens, patches)
    m.set(1)
    choice = choices(tokens, 2)
    m.run(**choice)
    h = m.table.double()[m.ids.long().clamp(min=0)] * 2
    z = m.features.double() @ m.projector.double().t() + m.bias.double()
    h[:patches] = 0.5 * z * torch.erfc(-z / math.sqrt(2))
    assert ((m.h.double() - h).abs() <= 2.0 ** -7 * h.abs() + 1e-3).all()
    y = h / (h.square().mean(1, keepdim=True) + EPS).sqrt() * m.norm.double()
    logits = y @ m.head.double().t()
    off = 5 * 2.0 ** -8 * y.norm(dim=1, keepdim=True) * m.head.double().norm(dim=1)
    assert ((m.logits.double() - logits).abs() <= off).all()
    again, logprob = torch.empty_like(m.token), torch.empty_like(m.logprob)
    B.qail_sample(m.logits.clone(), m.u, again, logprob=logprob, **choice)
    assert torch.equal(again, m.token) and torch.equal(logprob, m.logprob)
    greedy = choice["temperature"] == 0
    top = m.logits.max(1).values
    assert torch.equal(m.logits.gather(1, m.token.long()[:, None])[:, 0][greedy], top[greedy])


def test_captured_and_replayed(B):
    """One graph for other tokens and other random numbers, replayed with eager work between; every replay against the eager calls."""
    m, other = Model(B, 1000, 512, 136, 64, 20), Model(B, 1000, 512, 136, 64, 20)
    choice = choices(64, 3)
    m.set(1)
    m.run(**choice)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.run(**choice)
    for seed in range(5):
        m.set(seed)
        graph.replay()
        other.set(seed)
        other.run(**choice)
        torch.cuda.synchronize()
        assert torch.equal(m.token, other.token) and torch.equal(m.logits, other.logits) and torch.equal(m.logprob, other.logprob)


def test_two_streams(B):
    """Two models, each with buffers of its own, on two streams at once."""
    models = [Model(B, 1500, 512, 136, 200, 50) for _ in range(2)]
    want = []
    for i, m in enumerate(models):
        m.set(i)
        want.append(m.run().clone())
        m.token.fill_(-5)
    streams = [torch.cuda.Stream() for _ in models]
    torch.cuda.synchronize()
    for _ in range(5):
        for m, s in zip(models, streams):
            with torch.cuda.stream(s):
                m.run()
    torch.cuda.synchronize()
    assert all(torch.equal(m.token, w) for m, w in zip(models, want))


def training(B, m, teacher):
    """The loss of the logits and the gradients of the head, the norm's weight and the table, as the library gives them."""
    T, (vocab, hidden) = m.ids.numel(), m.table.shape
    loss, grad = torch.empty(1, device="cuda"), torch.empty_like(m.logits)
    B.qail_embed(m.table, m.ids, m.h, scale=2.0)
    B.qail_rmsnorm(m.h, m.norm, EPS, y=m.y)
    B.qail_w16a16_linear(m.d, m.y, m.logits, m.ws)
    B.qail_qbc_loss(m.logits, teacher, loss, grad, m.train_ws)
    B.qail_w16a16_backward(m.d, m.y, grad, m.train_ws, dx=m.dy, dweight=m.dhead)
    B.qail_rmsnorm_backward(m.h, m.norm, EPS, m.dy, m.dh, m.dnorm, m.train_ws)
    B.qail_embed_backward(m.ids, m.dh, m.dtable, m.train_ws, scale=2.0)
    return loss


def prepare_training(B, m):
    T, (vocab, hidden) = m.ids.numel(), m.table.shape
    m.dy, m.dh, m.dhead = torch.empty_like(m.h), torch.empty_like(m.h), torch.empty_like(m.head)
    m.dnorm, m.dtable = torch.empty(hidden, device="cuda"), torch.empty((vocab, hidden), device="cuda")
    m.train_ws = space(max(B.qail_w16a16_backward_workspace(m.d, T), B.qail_rmsnorm_backward_workspace(T, hidden), B.qail_embed_backward_workspace(vocab, hidden, T), 4 * T))


def test_the_way_back(B):
    """Gradients of the mean distance from a teacher's logits against automatic differentiation in 64 bits.  h, y, dy, dh and dz are rounded by 2^-8 at most each
    (2^-9 on average, of all their values at once: below 2^-8 of a gradient's norm per rounding on the way, of which there are up to six)."""
    m = Model(B, 400, 256, 64, 90, 0)
    m.set(4)
    prepare_training(B, m)
    teacher = normal((90, 400), 9, dtype=torch.float32)
    loss = training(B, m, teacher)
    table, norm, head = (t.double().requires_grad_() for t in (m.table, m.norm, m.head))
    h = 2 * table[m.ids.long()]
    y = h / (h.square().mean(1, keepdim=True) + EPS).sqrt() * norm
    want = (y @ head.t() - teacher.double()).norm(dim=1).mean()
    want.backward()
    assert abs(loss.item() - want.item()) <= 2.0 ** -7 * want.item()
    for got, exact in ((m.dhead, head.grad), (m.dnorm, norm.grad), (m.dtable, table.grad)):
        assert ((got.double() - exact).norm() / exact.norm()).item() <= 6 * 2.0 ** -8


def test_the_way_back_captured(B):
    m = Model(B, 400, 256, 64, 5000, 0)        # several tiles of tokens
    m.set(1)
    prepare_training(B, m)
    teacher = normal((5000, 400), 9, dtype=torch.float32)
    training(B, m, teacher)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        training(B, m, teacher)
    for seed in (1, 2, 3):
        m.set(seed)
        m.dtable.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (m.dhead, m.dnorm, m.dtable)]
        training(B, m, teacher)
        assert all(torch.equal(a, b) for a, b in zip(got, (m.dhead, m.dnorm, m.dtable)))


def test_the_example_draws_the_same_with_and_without_a_graph(S):
    m = S.Decoder(**SIZES)
    choice = dict(temperature=0.9, top_k=50, top_p=0.95, min_p=0.01)
    out, _ = S.serve(m, PROMPTS, [2, -1, 0], 8, graph=True, choice=choice, seed=5)
    again, _ = S.serve(m, PROMPTS, [2, -1, 0], 8, graph=False, choice=choice, seed=5)
    assert torch.equal(out, again) and out.min() >= 0
    greedy, _ = S.serve(m, PROMPTS, [2, -1, 0], 8)
    first, _ = S.serve(m, PROMPTS, [2, -1, 0], 8, choice=dict(temperature=1.0, top_k=1))
    assert torch.equal(greedy, first)


def test_the_example_trains_its_embeddings(S):
    """Rows without a token have no gradient, the others that of the loss: against automatic differentiation in 64 bits, bounds as above."""
    m = S.Decoder(**SIZES)
    ids = (torch.arange(40, device="cuda") % 7 * 11).to(torch.int32)
    teacher = normal((40, 300), 2, dtype=torch.float32)
    loss, dtable = S.embedding_gradient(m, ids, teacher)
    table = m.embedding.double().requires_grad_()
    h = table[ids.long()]
    want = ((h / (h.square().mean(1, keepdim=True) + EPS).sqrt() * m.last.double()) @ m.head.double().t() - teacher.double()).norm(dim=1).mean()
    want.backward()
    assert abs(loss - want.item()) <= 2.0 ** -7 * want.item()
    assert ((dtable.double() - table.grad).norm() / table.grad.norm()).item() <= 6 * 2.0 ** -8
    assert dtable.abs().amax(1).count_nonzero().item() == 7


def test_large_tiles_captured(B):
    """Products whose tiles need the opt-in for large LDS blocks, and shares of the contraction that pass through the workspace, in a graph."""
    cases = [(2056, 1024, 512), (1030, 2048, 2048), (700, 256, 4096)]
    held = []
    for i, (M, N, K) in enumerate(cases):
        w, b = normal((N, K), i, K ** -0.5), normal((N,), i + 1)
        d = B.make_w16a16(w, b, "silu")
        x, dy = normal((M, K), i + 2), normal((M, N), i + 3)
        out = dict(y=torch.empty((M, N), dtype=BF16, device="cuda"), z=torch.empty((M, N), dtype=BF16, device="cuda"), dx=torch.empty_like(x),
                   dweight=torch.empty((N, K), dtype=BF16, device="cuda"), dbias=torch.empty(N, device="cuda"))
        held.append(((d, w, b), x, dy, out, space(max(B.qail_w16a16_workspace(d, M), B.qail_w16a16_backward_workspace(d, M)))))

    def run():
        for (d, *_), x, dy, o, ws in held:
            B.qail_w16a16_linear(d, x, o["y"], ws, z=o["z"])
            B.qail_w16a16_backward(d, x, dy, ws, z=o["z"], dx=o["dx"], dweight=o["dweight"], dbias=o["dbias"])

    run()
    want = [{k: v.clone() for k, v in h[3].items()} for h in held]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for h in held:
            for v in h[3].values():
                v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(h[3][k], w[k]) for h, w in zip(held, want) for k in w)


def test_infinities_stay_in_their_rows(B):
    """An infinity or NaN in a row of x, or in a row of W, reaches that row (column) of the outputs alone, behind the end of K and N too."""
    for M, N, K in ((5, 70, 72), (130, 257, 264), (300, 72, 1000)):
        x, w = normal((M, K), 1), normal((N, K), 2)
        x[3, K - 1], w[7, K - 2] = float("inf"), float("nan")
        d = B.make_w16a16(w)
        y = torch.empty((M, N), device="cuda")
        B.qail_w16a16_linear(d, x, y, space(B.qail_w16a16_workspace(d, M)))
        bad = ~y.isfinite()
        assert bad[3].all() and bad[:, 7].all() and bad.sum().item() == N + M - 1
        dy = normal((M, N), 3)
        dy[2, N - 1] = float("inf")
        w = normal((N, K), 2)
        d = B.make_w16a16(w)
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(N, device="cuda")
        x = normal((M, K), 1)
        B.qail_w16a16_backward(d, x, dy, space(B.qail_w16a16_backward_workspace(d, M)), dx=dx, dweight=dw, dbias=db)
        assert (~dx.isfinite()).sum().item() == K and not dx[2].isfinite().any()
        assert (~dw.isfinite()).sum().item() == K and not dw[N - 1].isfinite().any()
        assert (~db.isfinite()).nonzero().flatten().tolist() == [N - 1]


def test_far_rows(B):
    """Tensors beyond 2^32 bytes: a table and its gradient, logits whose rows lie 2^31 values apart, and rows of a linear."""
    V, K = 70001, 32768
    table = torch.empty((V, K), dtype=BF16, device="cuda")
    for v in (0, 40000, 65535, 65536, V - 1):
        table[v] = normal((K,), v)
    ids = torch.tensor([V - 1, 0, 65536, 40000, 65535], dtype=torch.int32, device="cuda")
    h = torch.empty((5, K), dtype=BF16, device="cuda")
    B.qail_embed(table, ids, h)
    assert torch.equal(h, table[ids.long()])
    del table
    dtable = torch.empty((V, K), device="cuda")
    dtable[V - 2:] = 7
    B.qail_embed_backward(ids, h, dtable, space(B.qail_embed_backward_workspace(V, K, 5)))
    assert torch.equal(dtable[ids.long()], h.float()) and dtable[V - 2].abs().max() == 0
    del dtable
    wide = torch.empty((1 << 31) + (1 << 10), dtype=BF16, device="cuda")
    logits = wide.as_strided((2, 1000), (1 << 31, 1))
    logits.copy_(normal((2, 1000), 3))
    token, u = torch.empty(2, dtype=torch.int32, device="cuda"), torch.tensor([0.3, 0.6], device="cuda")
    B.qail_sample(logits, u, token)
    near = torch.empty_like(token)
    B.qail_sample(logits.contiguous(), u, near)
    assert torch.equal(token, near)
    del wide, logits
    M, K, N = (1 << 20) + 100, 4096, 8
    x, w = torch.zeros((M, K), dtype=BF16, device="cuda"), normal((N, K), 4, K ** -0.5)
    x[-200:] = normal((200, K), 5)
    d = B.make_w16a16(w)
    y = torch.empty((M, N), device="cuda")
    B.qail_w16a16_linear(d, x, y, space(B.qail_w16a16_workspace(d, M)))
    want = x[-200:].double() @ w.double().t()
    assert (y[-200:].double() - want).abs().max().item() <= (K + 2) * 2.0 ** -23 * (x[-200:].double().abs() @ w.double().abs().t()).max().item()
    assert y[:-200].abs().max() == 0


def test_plain_calls_give_the_same_by_either_way(B, monkeypatch):
    """The calls as C++ marshals them and as Python does, with every optional tensor; and what neither of them takes."""
    m = Model(B, 301, 64, 72, 40, 8)
    prepare_training(B, m)
    choice, z = choices(40, 4), torch.empty((8, 64), dtype=BF16, device="cuda")
    dp, dbias, dx = torch.empty_like(m.projector), torch.empty(64, device="cuda"), torch.empty_like(m.features)
    errors = torch.zeros(1, dtype=torch.int32, device="cuda")
    back = space(B.qail_w16a16_backward_workspace(m.p, 8))

    def everything():
        for t in (m.h, m.y, m.logits, m.token, m.logprob, z, dp, dbias, dx, m.dtable):
            t.fill_(3)
        m.set(9)
        m.ids[-2:] = torch.tensor([301, -7], dtype=torch.int32)
        errors.zero_()
        B.qail_w16a16_linear(m.p, m.features, m.h[:8], m.ws, residual=m.table[:8], z=z)
        B.qail_embed(m.table, m.ids, m.h, scale=2, errors=errors)
        B.qail_rmsnorm(m.h, m.norm, EPS, y=m.y)
        B.qail_w16a16_linear(m.d, m.y, m.logits, m.ws)
        B.qail_sample(m.logits, m.u, m.token, logprob=m.logprob, errors=errors, **choice)
        B.qail_w16a16_backward(m.p, m.features, m.h[:8], back, z=z, dx=dx, dweight=dp, dbias=dbias)
        B.qail_embed_backward(m.ids, m.h, m.dtable, m.train_ws, scale=0.5, accumulate=True, errors=errors)
        return [t.clone() for t in (m.h, m.logits, m.token, m.logprob, z, dp, dbias, dx, m.dtable, errors)]

    native = everything()
    assert native[-1].item() >= 2 and (m.token >= 0).all()
    for name in ("_embed_native", "_embed_backward_native", "_w16a16_native", "_w16a16_backward_native", "_sample_native"):
        assert getattr(B, name) is not B._not_plain
        monkeypatch.setattr(B, name, B._not_plain)
    assert all(torch.equal(a, b) for a, b in zip(native, everything()))
    for undo in (False, True):
        if undo:
            monkeypatch.undo()
        with pytest.raises(ValueError):
            B.qail_embed(m.table, m.ids, m.h.t().contiguous().t())
        with pytest.raises(ValueError):
            B.qail_embed_backward(m.ids, m.h[:-1], m.dtable, m.train_ws)
        with pytest.raises(ValueError):
            B.qail_w16a16_linear(m.d, m.y, m.logits.cpu(), m.ws)
        with pytest.raises(ValueError):
            B.qail_w16a16_backward(m.p, m.features.float(), m.h[:8], back, z=z, dweight=dp)
        with pytest.raises(ValueError):
            B.qail_sample(m.logits.t(), m.u, m.token)


@pytest.mark.parametrize("plain", [True, False])
def test_linears_take_rows_in_any_number_of_dimensions(B, monkeypatch, plain):
    """Frames x patches x width is that many rows, by either way of marshalling."""
    if not plain:
        for name in ("_w16a16_native", "_w16a16_backward_native"):
            monkeypatch.setattr(B, name, B._not_plain)
    g = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    F, P, K, N = 3, 17, 64, 40
    x, w, b, dy = new(F, P, K), new(N, K), new(N), new(F, P, N)
    d = B.make_w16a16(w, b, "silu")

    def run(x, dy):
        M = F * P
        y, z = (torch.full((*x.shape[:-1], N), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ws = torch.empty(max(B.qail_w16a16_workspace(d, M), B.qail_w16a16_backward_workspace(d, M)), dtype=torch.uint8, device="cuda")
        B.qail_w16a16_linear(d, x, y, ws, z=z)
        out = [torch.full_like(x, float("nan")), torch.full_like(w, float("nan")), torch.full((N,), float("nan"), device="cuda")]
        B.qail_w16a16_backward(d, x, dy, ws, z=z, dx=out[0], dweight=out[1], dbias=out[2])
        return [y, z, *out]

    for a, e in zip(run(x, dy), run(x.view(F * P, K), dy.view(F * P, N))):
        assert torch.equal(a.flatten(), e.flatten()) and torch.isfinite(a).all()
    one = B.make_w16a16(w[:1].contiguous())       # one output: its gradient may be a list of numbers
    dx, flat = torch.empty((F * P, K), dtype=torch.bfloat16, device="cuda"), torch.empty((F * P, K), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.qail_w16a16_backward_workspace(one, F * P), dtype=torch.uint8, device="cuda")
    B.qail_w16a16_backward(one, None, dy[..., :1].contiguous(), ws, dx=dx)
    B.qail_w16a16_backward(one, None, dy[..., 0].flatten().contiguous(), ws, dx=flat)
    assert torch.equal(dx, flat)
