"""The functions of the 16-bit linears' epilogue far out: infinities, NaN, and values whose functions are small."""
import math

import pytest
import torch

from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu
BF16, INF, NAN = torch.bfloat16, float("inf"), float("nan")
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")


@pytest.fixture(scope="module")
def B():
    return ensure_built()


def space(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda").fill_(0xFF) if n else None


def plain(name, z):
    """The definitions, in 64 bits."""
    if name == "gelu":
        return z * (1 + torch.erf(z / math.sqrt(2))) / 2
    if name == "gelu_tanh":
        return z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))) / 2
    return {"none": z, "relu": torch.where(z < 0, 0.0, z), "silu": z / (1 + torch.exp(-z))}[name]


@pytest.mark.parametrize("activation", ACTIVATIONS)
@pytest.mark.parametrize("out", [BF16, torch.float32])
@pytest.mark.parametrize("how", ["z", "bias", "sum"])
def test_an_infinity_is_what_the_function_makes_of_it(B, activation, out, how):
    """In whole groups of eight columns and behind them, in rows of few and of many blocks' tiles: of x, of the bias, and of a sum that has no fp32 number."""
    for M, N in ((3, 11), (140, 261)):
        x, w, b = torch.zeros((M, 8), dtype=BF16, device="cuda"), torch.ones((N, 8), dtype=BF16, device="cuda"), torch.zeros(N, dtype=BF16, device="cuda")
        x[:, 0] = 1
        at = [0, 5, N - 3, N - 2, N - 1]
        if how == "z":
            x[0, 0], x[1, 0], x[M - 1, 0] = INF, NAN, -INF
        elif how == "bias":
            b[at] = torch.tensor([INF, -INF, NAN, INF, -INF], dtype=BF16, device="cuda")
        else:
            w[at, 0] = torch.tensor([3e38, -3e38, 3e38, -3e38, 3e38], dtype=BF16, device="cuda")
            w[at, 1] = w[at, 0]
            x[:, 1] = 1
        z = x[:, :1].float() * w[:, 0].float() + x[:, 1:2].float() * w[:, 1].float() + b.float()
        assert not torch.isfinite(z).all()
        y = torch.full((M, N), 7.0, dtype=out, device="cuda")
        d = B.make_w16a16(w, b, activation)
        B.qail_w16a16_linear(d, x, y, space(B.qail_w16a16_workspace(d, M)))
        want = plain(activation, z.double())
        assert torch.equal(torch.isnan(y), torch.isnan(want)), activation
        assert torch.equal(y[torch.isinf(want)].double(), want[torch.isinf(want)]) and torch.isfinite(y[torch.isfinite(want)]).all(), activation
        off = (2.0 ** -7 if out == BF16 else 2.0 ** -20) * want.abs() + 2.0 ** -24
        assert ((y.double() - want).abs() <= off)[torch.isfinite(want)].all(), activation


# Of the function's value, far from 0: the exact GELU for bf16 outputs takes a tail good to 2^-14.7 and an exponential of an argument in one part, up to 126 with three roundings of 2^-24 of
# itself (2^-16.5 of the exponential); the argument of tanh-GELU's exponential, up to 88, has four (2^-15.5).
GOOD_TO = {"gelu": 2.0 ** -20, "gelu_tanh": 2.0 ** -15, "silu": 2.0 ** -20}


@pytest.mark.parametrize("activation, low", [("gelu", -14.0), ("gelu_tanh", -10.5), ("silu", -95.0)])
@pytest.mark.parametrize("out", [BF16, torch.float32])
def test_small_values_are_good_to_a_share_of_themselves(B, activation, low, out):
    """Down to 2^-119: below, reciprocals and exponentials have no normal numbers.  All columns of a row are the same sum, and the last seven, which are written one by one, have the
    values of the first eight."""
    z = torch.cat((torch.linspace(low, 8, 6001), -torch.logspace(-30, 1, 500))).cuda().to(BF16)
    M, N = z.numel(), 15
    w = torch.zeros((N, 8), dtype=BF16, device="cuda")
    w[:, 0] = 1
    x = torch.zeros((M, 8), dtype=BF16, device="cuda")
    x[:, 0] = z
    y = torch.full((M, N), NAN, dtype=out, device="cuda")
    d = B.make_w16a16(w, None, activation)
    B.qail_w16a16_linear(d, x, y, space(B.qail_w16a16_workspace(d, M)))
    assert torch.equal(y, y[:, :1].expand(-1, N))
    t = z.double()
    if activation == "gelu":
        want = t * torch.erfc(-t / math.sqrt(2)) / 2
    else:
        want = t / (1 + torch.exp(-t if activation == "silu" else -math.sqrt(8 / math.pi) * (t + 0.044715 * t ** 3)))
    good = 2.0 ** -14 if activation == "gelu" and out == BF16 else GOOD_TO[activation]
    off = (good + (2.0 ** -8 if out == BF16 else 2.0 ** -24)) * want.abs() + 2.0 ** -119
    assert ((y[:, 0].double() - want).abs() <= off).all()
