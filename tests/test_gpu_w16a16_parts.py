"""The gradients' products of the 16-bit linears have dz in two bf16 parts, unless the caller asks for a rounded one.

Whole numbers of at most 15 bits are the sum of two bf16 numbers, and sums of them below 2^24 are exact in fp32 in any order: with x and W of 1 and -1 the gradients are those of
whole numbers, rounded once to bf16.  Elsewhere the first part is off by 2^-8 of dz at most and the second one by 2^-8 of that, which is 2^-16 of dz."""
import math

import pytest
import torch

from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu
BF16, INF, NAN = torch.bfloat16, float("inf"), float("nan")


@pytest.fixture(scope="module")
def B():
    return ensure_built()


def normal(shape, seed, std=1.0, dtype=BF16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def signs(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randint(0, 2, shape, generator=g, device="cuda") * 2 - 1).to(BF16)


def backward(B, x, w, dy, activation="none", z=None, **more):
    d = B.make_w16a16(w, None, activation, **more)
    ws = torch.empty(B.qail_w16a16_backward_workspace(d, dy.shape[0]), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = dict(dx=torch.full_like(x, NAN), dweight=torch.full_like(w, NAN), dbias=torch.full((w.shape[0],), NAN, device="cuda"))
    B.qail_w16a16_backward(d, x, dy, ws, z=z, **out)
    return out


SIZES = [(1, 1, 8), (3, 41, 200), (33, 264, 72), (129, 255, 1000), (289, 1024, 136), (16, 8192, 64), (640, 640, 640), (2056, 264, 72), (1100, 24, 16), (300, 2501, 1000),
         (5000, 65, 40), (2048, 2048, 2048), (2500, 2100, 2056), (289, 4096, 4096)]


@pytest.mark.parametrize("M, N, K", SIZES)
@pytest.mark.parametrize("activation", ["none", "relu"])
def test_whole_numbers_are_added_up_exactly(B, M, N, K, activation):
    bits = min(15, 24 - math.ceil(math.log2(max(M, N))))
    g = torch.Generator(device="cuda").manual_seed(M + N)
    dy = torch.randint(1 - 2 ** bits, 2 ** bits, (M, N), generator=g, device="cuda").float()
    x, w, z = signs((M, K), 1), signs((N, K), 2), signs((M, N), 3)
    out = backward(B, x, w, dy, activation, z if activation == "relu" else None)
    dz = dy.double() * (z > 0).double() if activation == "relu" else dy.double()
    assert torch.equal(out["dx"], (dz @ w.double()).to(BF16))
    assert torch.equal(out["dweight"], (dz.t().contiguous() @ x.double()).to(BF16))
    assert torch.equal(out["dbias"].double(), dz.sum(0))


@pytest.mark.parametrize("M, N, K", SIZES)
def test_a_rounded_dz_where_the_caller_asks_for_it(B, M, N, K):
    bits = min(15, 24 - math.ceil(math.log2(max(M, N))))
    g = torch.Generator(device="cuda").manual_seed(M + N)
    dy = torch.randint(1 - 2 ** bits, 2 ** bits, (M, N), generator=g, device="cuda").float()
    x, w = signs((M, K), 1), signs((N, K), 2)
    out = backward(B, x, w, dy, round_dz=True)
    dz = dy.to(BF16).double()
    assert torch.equal(out["dx"], (dz @ w.double()).to(BF16))
    assert torch.equal(out["dweight"], (dz.t().contiguous() @ x.double()).to(BF16))
    assert torch.equal(out["dbias"].double(), dy.double().sum(0))


def slope(name, z):
    if name == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    a = math.sqrt(8 / math.pi)
    v, dv = (z, 1.0) if name == "silu" else (a * (z + 0.044715 * z ** 3), a * (1 + 3 * 0.044715 * z * z))
    s = torch.sigmoid(v)
    return s + z * s * torch.sigmoid(-v) * dv


@pytest.mark.parametrize("activation", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M, N, K", [(40, 40, 72), (63, 65, 136)])
@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_gradients_have_their_own_rounding_alone(B, M, N, K, activation, dtype):
    """Slopes are good to 2^-20 of max(|z|, 1); an fp32 sum of 2 R products to 2 R + 2 halves of a step of 2^-23 of the sum of their sizes."""
    x, w, dy, z = normal((M, K), 1), normal((N, K), 2, K ** -0.5), normal((M, N), 3, dtype=dtype), normal((M, N), 4)
    out = backward(B, x, w, dy, activation, z)
    dz = dy.double() * slope(activation, z.double())
    off_z = 2.0 ** -20 * dy.double().abs() * z.double().abs().clamp(min=1) + 2.0 ** -16 * dz.abs()
    for name, a, off, b, R in (("dx", dz, off_z, w, N), ("dweight", dz.t().contiguous(), off_z.t().contiguous(), x, M)):
        want = a @ b.double()
        off = (2 * R + 2) * 2.0 ** -23 * (a.abs() @ b.double().abs()) * (1 + 2.0 ** -8) + off @ b.double().abs()
        over = (out[name].double() - want).abs() - off - 2.0 ** -8 * (want.abs() + off)
        assert over.max().item() <= 0, (name, over.max().item())


def same_where_not_finite(got, want):
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.isinf(got), torch.isinf(want)) and torch.equal(got[torch.isinf(want)].sign().double(), want[torch.isinf(want)].sign())
    finite = torch.isfinite(want)
    assert finite.any()
    assert ((got.double() - want)[finite].abs() <= 2.0 ** -7 * want[finite].abs() + 2.0 ** -8).all()


@pytest.mark.parametrize("M, N, K", [(33, 264, 72), (289, 1024, 136), (20, 8192, 64), (700, 640, 640), (2048, 2056, 2048)])
def test_infinities_and_nan_are_those_of_the_product(B, M, N, K):
    """The second part of dz meets an infinity with any sign, or is 0 (a dy of whole numbers below 256): the product's is that of dz itself."""
    g = torch.Generator(device="cuda").manual_seed(M)
    dy = torch.randint(1, 1 << 10, (M, N), generator=g, device="cuda").float() * signs((M, N), 1).float()
    x, w = signs((M, K), 2), signs((N, K), 3)
    w[N // 3, 5], w[N // 2, 9], w[N - 1, 17] = INF, -INF, NAN
    x[M // 3, 3], x[M // 2, 11], x[M - 1, 21] = -INF, INF, NAN
    dy[M // 4, N // 5], dy[M // 5, N - 2] = INF, NAN
    out = backward(B, x, w, dy)

    def product(a, b):
        """Of matrices with a few infinities and NaN, whose terms are looked at one column at a time."""
        want = a.nan_to_num(0, 0, 0) @ b.nan_to_num(0, 0, 0)
        for i in (~torch.isfinite(a)).any(0).nonzero()[:, 0].tolist():
            rows = ~torch.isfinite(a[:, i])
            want[rows] += a[rows, i][:, None] * b[i][None]
        for i, k in (~torch.isfinite(b)).nonzero().tolist():
            want[:, k] += a[:, i] * b[i, k]
        return want

    same_where_not_finite(out["dx"], product(dy.double(), w.double()))
    same_where_not_finite(out["dweight"], product(dy.t().contiguous().double(), x.double()))
    rows = torch.isfinite(dy).all(0)
    assert torch.equal(out["dbias"].double()[rows], dy.double().sum(0)[rows]) and not torch.isfinite(out["dbias"][~rows]).any()


def test_a_dy_beyond_the_largest_bf16_number(B):
    """It is finite, and so are the gradients: the first part is the largest number of bf16 then."""
    dy = torch.zeros((5, 8), device="cuda")
    dy[1, 2], dy[3, 4] = 3.4e38, -3.402e38
    x, w = torch.full((5, 16), 2.0 ** -20, dtype=BF16, device="cuda"), torch.full((8, 16), 2.0 ** -10, dtype=BF16, device="cuda")
    out = backward(B, x, w, dy)
    for got, want in ((out["dx"], dy.double() @ w.double()), (out["dweight"], dy.double().t().contiguous() @ x.double())):
        assert torch.equal(got, want.to(BF16))
