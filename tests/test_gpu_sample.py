"""Sampling against its definition in whole numbers: the same tokens, log-probabilities to fp32."""
import math

import numpy as np
import pytest
import torch

from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    return ensure_built()


def reference(x, u, t, k, p, m):
    """Token and logprob of one row by the definition: weights are whole multiples of 2^-44, sums exact."""
    order = np.argsort(-x, kind="stable")
    if t == 0:
        return int(order[0]), 0.0
    with np.errstate(invalid="ignore"):
        down = (x[order] - x[order[0]]) / t
    w = np.floor(np.exp(down) * 2.0 ** 44 + 0.5).astype(np.int64)
    n = len(x)
    if k > 0:
        n = min(n, k)
    if p < 1:
        upto = np.cumsum(w[:n])
        n = 1 + int(np.searchsorted(upto, max(1, math.ceil(float(p) * float(upto[-1])))))
    if m > 0:
        n = min(n, max(1, int((down >= math.log(float(m))).sum())))
    kept, w, down = order[:n], w[:n], down[:n]
    by = np.argsort(kept)
    upto = np.cumsum(w[by])
    i = int(np.searchsorted(upto, int(float(u) * float(upto[-1])), side="right"))
    return int(kept[by[i]]), float(down[by[i]] - math.log(float(upto[-1]) / 2.0 ** 44))


def check(B, logits, u, t=None, k=None, p=None, m=None):
    """logprob: two roundings of 2^-24 of it, one of the value near zero by 64-bit logarithms."""
    R = logits.shape[0]
    dev = lambda v, dtype: None if v is None else torch.tensor(v, dtype=dtype, device="cuda")  # noqa: E731
    t32, p32, m32, u32 = (dev(v, torch.float32) for v in (t, p, m, u))
    token, logprob = torch.full((R,), -7, dtype=torch.int32, device="cuda"), torch.full((R,), float("nan"), device="cuda")
    errors = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.qail_sample(logits, u32, token, logprob=logprob, temperature=t32, top_k=dev(k, torch.int32), top_p=p32, min_p=m32, errors=errors)
    assert errors.item() == 0
    x = logits.double().cpu().numpy()
    value = lambda v, r, off: off if v is None else v[r].item()  # noqa: E731
    want = [reference(x[r], u32[r].item(), value(t32, r, 1.0), 0 if k is None else k[r], value(p32, r, 1.0), value(m32, r, 0.0)) for r in range(R)]
    assert token.tolist() == [w[0] for w in want]
    for got, (_, lp) in zip(logprob.tolist(), want):
        assert abs(got - lp) <= 2.0 ** -23 * abs(lp) + 1e-9, (got, lp)
    again = torch.empty_like(token)
    B.qail_sample(logits, u32, again, temperature=t32, top_k=dev(k, torch.int32), top_p=p32, min_p=m32)
    assert torch.equal(token, again)


def rows(R, V, seed, dtype, width=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((R, V), generator=g, device="cuda") * width).to(dtype)


def randoms(R, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.rand((R,), generator=g).tolist()


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 64, 65, 511, 512, 513, 1000, 8191, 8192, 8193, 32000, 50001, 131072, 1 << 18])
def test_lengths(B, V, dtype):
    R = 6
    x = rows(R, V, V, dtype)
    check(B, x, randoms(R, V))
    check(B, x, randoms(R, V + 1), [0.7, 1.0, 1.3, 0.0, 0.2, 5.0], [0, 3, 50, 5, V, V + 1], [0.9, 1.0, 0.5, 0.9, 0.99, 0.95], [0.0, 0.1, 0.0, 0.5, 0.01, 0.3])


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_choices(B, dtype):
    """Every combination of a temperature and the three filters, each a row of one call."""
    choices = [(t, k, p, m) for t in (0.0, 0.05, 0.8, 1.0, 2.0, 50.0) for k in (-3, 0, 1, 2, 40, 5000) for p in (-1.0, 0.0, 0.3, 0.95, 1.0, 2.0) for m in (-0.5, 0.0, 0.05, 1.0, 1.5)]
    t, k, p, m = zip(*choices)
    x = rows(len(choices), 1500, 1, dtype)
    check(B, x, randoms(len(choices), 2), t, k, [v for v in p], m)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_equal_logits_and_masks(B, dtype):
    V = 3000
    x = rows(14, V, 5, dtype)
    x[0] = 0.0                                        # all equal
    x[1, ::2], x[1, 1::2] = 0.0, -0.0                 # equal as well
    x[2] = x[2].round()                               # many equal ones
    x[3] = -math.inf
    x[3, 1234] = -50.0                                # one token is left
    x[4, :2900] = -math.inf
    x[5] = -math.inf
    x[5, [7, 2999]] = torch.tensor([1.0, 1.0], dtype=dtype, device="cuda")
    x[6] = -1e30
    x[6, 5] = 1e30
    x[7] = 3.0e38
    x[8] = torch.where(torch.arange(V, device="cuda") % 3 == 0, 3.0, -3.0).to(dtype)
    x[9] = torch.linspace(0, -40, V, device="cuda").to(dtype)     # down to weights of zero
    x[10] = x[10] * 1e-30
    x[11, 1:] = torch.finfo(dtype).min                            # a mask of the type's lowest value
    for seed in range(4):
        n = 14
        check(B, x, randoms(n, seed))
        check(B, x, [0.0] * n, [1.0] * n, None, [0.9] * n)
        check(B, x, [1 - 2.0 ** -24] * n, [1.0] * n, [100] * n, [0.9] * n)
        check(B, x, randoms(n, 10 + seed), [0.9] * n, [30] * n, [0.5] * n, [0.2] * n)
        check(B, x, randoms(n, 20 + seed), None, None, [0.7] * n)
        check(B, x, randoms(n, 30 + seed), None, [1500] * n)


def test_rows_that_cannot_be_drawn_from(B):
    V = 700
    bad = [lambda x: x.fill_(-math.inf), lambda x: x[3:4].fill_(float("nan")), lambda x: x[699:].fill_(math.inf), lambda x: x.fill_(float("nan"))]
    for dtype in (BF16, torch.float32):
        x = rows(2 * len(bad), V, 3, dtype)
        for i, spoil in enumerate(bad):
            spoil(x[2 * i])
        token, logprob = torch.full((8,), 5, dtype=torch.int32, device="cuda"), torch.zeros(8, device="cuda")
        errors = torch.zeros(1, dtype=torch.int32, device="cuda")
        u = torch.tensor(randoms(8, 4), device="cuda")
        B.qail_sample(x, u, token, logprob=logprob, errors=errors)
        assert errors.item() == 4 and token[::2].tolist() == [-1] * 4 and logprob[::2].isnan().all()
        want = [reference(x[i].double().cpu().numpy(), u[i].item(), 1.0, 0, 1.0, 0.0)[0] for i in (1, 3, 5, 7)]
        assert token[1::2].tolist() == want
    x = rows(9, V, 3, BF16)
    col = lambda *v: torch.tensor(v, device="cuda")  # noqa: E731
    t = col(-1.0, float("nan"), math.inf, 0.0, 1.0, 1.0, 1.0, 1.0, 1.0)
    p = col(1.0, 1.0, 1.0, 1.0, float("nan"), 1.0, 1.0, 1.0, 0.9)
    m = col(0.0, 0.0, 0.0, 0.0, 0.0, float("nan"), 0.0, 0.0, 0.0)
    u = col(0.5, 0.5, 0.5, 9.0, 0.5, 0.5, 1.0, -0.1, 0.5)
    token, errors = torch.zeros(9, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.qail_sample(x, u, token, temperature=t, top_p=p, min_p=m, errors=errors)
    assert [v < 0 for v in token.tolist()] == [True, True, True, False, True, True, True, True, False] and errors.item() == 7
    B.qail_sample(x[:0], u[:0], token[:0])


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_rows_of_wider_tensors(B, dtype):
    wide = rows(5, 4096, 9, dtype)
    check(B, wide[:, 64:1064], randoms(5, 1), [0.8] * 5, [100] * 5, [0.9] * 5)
    odd = rows(5, 1001, 9, dtype)                      # rows that begin anywhere
    check(B, odd, randoms(5, 2), [0.8] * 5, None, [0.9] * 5)
    check(B, odd[:, :999], randoms(5, 3))
    check(B, wide[::2, :777], randoms(3, 4), None, [20] * 3)
    for V in (1, 3, 5, 8187, 8189, 8193, 32763, 32767, 40003, (1 << 18) - 1):   # rows that skip 0 to 7 values, whose neighbours would be drawn
        x = rows(9, V, V, dtype)
        x[4] += 30
        check(B, x, randoms(9, V), [1.0] * 8 + [0.0], [0, 7, 0, V, 2, 0, 0, 1, 0], [1.0, 0.9, 0.8, 1.0, 1.0, 0.99, 1.0, 1.0, 1.0], [0.0] * 6 + [0.1, 0.0, 0.0])


def test_temperatures_next_to_the_steps_of_the_logits(B):
    """Neighbouring logits whose distance is tens of temperatures: the next one's weight is around the least that counts, and below."""
    for most in (1e6, -1e6, 37.0):
        step = np.spacing(np.float32(most))
        x = torch.tensor([[most - i * step for i in range(40)]], dtype=torch.float32, device="cuda").expand(60, -1).contiguous()
        t = [abs(float(step)) / d for d in np.linspace(0.5, 60.0, 60)]
        for k, p in ((None, None), ([3] * 60, None), (None, [0.97] * 60), ([3] * 60, [0.97] * 60)):
            check(B, x, randoms(60, 8), t, k, p)
            check(B, x, [1 - 2.0 ** -24] * 60, t, k, p)
    check(B, rows(4, 500, 1, torch.float32), randoms(4, 1), [1e-45, 1e-38, 3e38, 1e30], [0, 20, 0, 20], [0.9] * 4)


def test_frequencies(B):
    """64 equal steps of u over one row: the tokens come as often as their probabilities say, to one step."""
    p = torch.tensor([0.5, 0.25, 0.125, 0.0625, 0.0625], device="cuda")
    x = p.log()[None].expand(64, -1).contiguous()
    u = (torch.arange(64, device="cuda") + 0.5) / 64
    token = torch.empty(64, dtype=torch.int32, device="cuda")
    B.qail_sample(x, u, token)
    assert torch.bincount(token.long(), minlength=5).tolist() == [32, 16, 8, 4, 4]
