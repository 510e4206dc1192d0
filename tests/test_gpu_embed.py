"""The lookup of embeddings and its gradient against plain forms: the lookup bit for bit, the gradient against sums in 64 bits."""
import pytest
import torch

from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    return ensure_built()


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(shape, seed, dtype=BF16):
    return torch.randn(shape, generator=rng(seed), device="cuda").to(dtype)


def numbers(T, V, seed, holes=0):
    ids = torch.randint(0, V, (T,), generator=rng(seed), device="cuda", dtype=torch.int32)
    if holes:
        ids[torch.randperm(T, generator=rng(seed + 1), device="cuda")[:holes]] = -1
    return ids


@pytest.mark.parametrize("T, V, K, scale, holes", [
    (1, 1, 8, 1.0, 0), (7, 100, 64, 2.5, 2), (16, 2000, 4096, 1.0, 0), (33, 50, 2056, -0.3, 5), (5, 9, 1304, 64.0, 5), (300, 77, 24, 1.0, 30), (3, 11, 16384, 1.0, 0),
    (2000, 3, 136, 0.1, 7)])
def test_lookup(B, T, V, K, scale, holes):
    table, ids, before = normal((V, K), 1), numbers(T, V, 2, holes), normal((T, K), 3)
    h, errors = before.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.qail_embed(table, ids, h, scale=scale, errors=errors)
    want = torch.where((ids < 0)[:, None], before, (table.float()[ids.long().clamp(min=0)] * scale).to(BF16))
    assert torch.equal(h, want) and errors.item() == 0


def test_lookup_of_tokens_that_are_not_in_the_table(B):
    ids = torch.tensor([0, 10, -1, -(1 << 31), (1 << 31) - 1, 9, 11], dtype=torch.int32, device="cuda")
    table, before = normal((10, 72), 1), normal((7, 72), 2)
    h, errors = before.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.qail_embed(table, ids, h, errors=errors)
    assert torch.equal(h[[0, 5]], table[[0, 9]]) and torch.equal(h[[2, 3]], before[[2, 3]]) and h[[1, 4, 6]].abs().max() == 0
    assert errors.item() >= 1
    B.qail_embed(table, ids, h)    # without a counter
    B.qail_embed(table, ids[:0], h[:0])
    torch.cuda.synchronize()


def check_gradient(B, ids, V, K, scale, seed, accumulate=False):
    """Sums of n terms in fp32: each addition is off by 2^-24 of a partial sum at most, the product with the scale and the addition to what was there by
    as much of the result: (n + 2) 2^-24 of the sum of magnitudes."""
    T = ids.numel()
    dh = normal((T, K), seed)
    held = (ids >= 0) & (ids < V)
    dh[~held] = float("nan")       # rows that belong to no token
    before = normal((V, K), seed + 1, torch.float32)
    out = before.clone() if accumulate else torch.full((V, K), float("nan"), device="cuda")
    errors = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.qail_embed_backward_workspace(V, K, T), dtype=torch.uint8, device="cuda").fill_(0xFF)
    B.qail_embed_backward(ids, dh, out, ws, scale=scale, accumulate=accumulate, errors=errors)
    place = ids[held].long()
    rows = dh[held].double() * scale
    want = torch.zeros((V, K), dtype=torch.float64, device="cuda").index_add_(0, place, rows)
    size = torch.zeros((V, K), dtype=torch.float64, device="cuda").index_add_(0, place, rows.abs())
    n = torch.bincount(place, minlength=V).double()[:, None]
    if accumulate:
        want, size = want + before.double(), size + before.double().abs()
        assert torch.equal(out[n[:, 0] == 0], before[n[:, 0] == 0])
    off = (out.double() - want).abs() - (n + 2) * 2.0 ** -24 * size
    assert off.max().item() <= 0, off.max().item()
    assert (errors.item() > 0) == bool((ids >= V).any())
    again = before.clone() if accumulate else torch.empty_like(out)
    B.qail_embed_backward(ids, dh, again, ws, scale=scale, accumulate=accumulate)
    assert torch.equal(out, again)


@pytest.mark.parametrize("T, V, K, scale, holes", [
    (1, 1, 8, 1.0, 0), (1, 255, 8, 1.0, 0), (5, 256, 72, 2.0, 1), (32, 3, 1024, 1.0, 0), (33, 1, 1032, 1.0, 0), (63, 2, 64, -0.5, 0), (64, 2, 64, 1.0, 3),
    (1000, 7, 200, 1.0, 100), (4096, 65, 64, 1.0, 0), (4096, 70000, 16, 1.0, 9), (4097, 65, 64, 0.25, 11), (4097, 300, 40, 1.0, 0), (9000, 70000, 8, 1.0, 0),
    (12289, 5, 136, 1.0, 12000), (30000, 2000, 48, 3.0, 17), (65536, 300, 8, 1.0, 0), (65537, 300, 8, 1.0, 5), (70001, 70000, 8, 1.0, 5), (257, 1000, 4104, 1.0, 0), (5000, 1, 8, 1.0, 4999),
    (2, 1, 8, 1.0, 1), (255, 3, 72, 1.0, 0), (256, 40, 264, 1.0, 100), (256, 1 << 23, 8, 1.0, 3)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(B, T, V, K, scale, holes, accumulate):
    check_gradient(B, numbers(T, V, T + V, holes), V, K, scale, 5, accumulate)


@pytest.mark.parametrize("T", [40, 4096, 8200, 66000])
def test_gradient_of_a_common_token(B, T):
    """Most rows are one token's, as padding's are; it begins and ends inside parts and at their edges."""
    for first in (0, 1, 31, 32, 33):
        ids = torch.full((T,), 3, dtype=torch.int32, device="cuda")
        ids[:first] = 1
        ids[-3:] = torch.tensor([7, 2, 5], dtype=torch.int32, device="cuda")
        check_gradient(B, ids[torch.randperm(T, generator=rng(first), device="cuda")], 9, 264, 1.0, first)


def test_gradient_without_tokens_and_with_bad_ones(B):
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    out = torch.ones((5, 64), device="cuda")
    ws = torch.empty(B.qail_embed_backward_workspace(5, 64, 0), dtype=torch.uint8, device="cuda")
    B.qail_embed_backward(none, normal((0, 64), 1), out, ws, accumulate=True)
    assert out.min() == 1
    B.qail_embed_backward(none, normal((0, 64), 1), out, ws)
    assert out.abs().max() == 0
    for T in (50, 5000):
        ids = numbers(T, 20, 3)
        ids[::7], ids[3] = 20, (1 << 31) - 1
        check_gradient(B, ids, 20, 64, 1.0, 4)
        check_gradient(B, torch.full_like(ids, -1), 20, 64, 1.0, 4)


def test_gradient_agrees_with_differences(B):
    """Of the loss sum(h * c): the lookup is linear in the table, so a difference over 2 divided by 2 is exact up to the roundings of h (2^-8 of its values, 8 of them)."""
    V, K, T = 6, 8, 9
    table, ids, c = normal((V, K), 1), numbers(T, V, 2, 2), normal((T, K), 3)
    dtable, ws = torch.empty((V, K), device="cuda"), torch.empty(B.qail_embed_backward_workspace(V, K, T), dtype=torch.uint8, device="cuda")
    B.qail_embed_backward(ids, c, dtable, ws, scale=1.5)

    def loss(t):
        h = torch.zeros((T, K), dtype=BF16, device="cuda")
        B.qail_embed(t, ids, h, scale=1.5)
        return (h.double() * c.double()).sum().item(), (h.double() * c.double()).abs().sum().item()

    for v in range(V):
        t = table.clone()
        t[v, 3] += 2
        step = (t[v, 3].double() - table[v, 3].double()).item()
        (a, sa), (b, sb) = loss(t), loss(table)
        assert abs((a - b) / step - dtable[v, 3].item()) <= 2.0 ** -8 * (sa + sb) / abs(step) + 1e-6
