"""Linears with 16-bit weights, their epilogue and their gradients, against products in 64 bits.

A product's fp32 sum of R terms is off by at most R + 2 halves of a step of 2^-23 (whatever the order of the sum) of S, the sum of the terms' magnitudes; functions
of z are evaluated to 2^-20 of max(|z|, 1) and have slopes of at most 1.13 (and curvatures of at most 1.13 as well), GELU for bf16 outputs to 2^-14.7 of its tail; a bf16 result is rounded by 2^-8 of itself at most."""
import math

import pytest
import torch

from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")


@pytest.fixture(scope="module")
def B():
    return ensure_built()


def normal(shape, seed, std=1.0, dtype=BF16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def function(name, z):
    """act(z) and its slope in 64 bits."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "gelu":
        p = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    a = math.sqrt(8 / math.pi)
    v, dv = (z, 1.0) if name == "silu" else (a * (z + 0.044715 * z ** 3), a * (1 + 3 * 0.044715 * z * z))
    s = torch.sigmoid(v)
    return z * s, s + z * s * torch.sigmoid(-v) * dv


def space(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda").fill_(0xFF) if n else None


def check_forward(B, M, N, K, activation="none", bias=False, residual=False, keep=False, out=BF16, seed=0, in_place=False):
    x, w = normal((M, K), seed), normal((N, K), seed + 1, K ** -0.5)
    b = normal((N,), seed + 2, 0.5) if bias else None
    r = normal((M, N), seed + 3) if residual else None
    y = r.clone() if in_place else torch.full((M, N), float("nan"), dtype=out, device="cuda")
    z = torch.full((M, N), float("nan"), dtype=BF16, device="cuda") if keep else None
    d = B.make_w16a16(w, b, activation)
    ws = space(B.qail_w16a16_workspace(d, M))
    B.qail_w16a16_linear(d, x, y, ws, residual=y if in_place else r, z=z)
    want_z = x.double() @ w.double().t() + (b.double() if bias else 0)
    off_z = (K + 2) * 2.0 ** -23 * (x.double().abs() @ w.double().abs().t() + (b.double().abs() if bias else 0))
    want = function(activation, want_z)[0]
    off = 1.13 * off_z + (2.0 ** -20 * want_z.abs().clamp(min=1) if activation not in ("none", "relu") else 0)
    if activation == "gelu" and out == BF16:
        # z times the share of the normal distribution beyond |z|, at most 0.17, is the part that the shorter form has to 2^-14.7
        off = off + 0.17 * 2.0 ** -14.7
    if residual:
        want = want + r.double()
        off = off + 2.0 ** -24 * want.abs()
    half = 2.0 ** -8 if out == BF16 else 2.0 ** -24
    over = (y.double() - want).abs() - off - half * (want.abs() + off)
    assert over.max().item() <= 0, (over.max().item(), over.argmax().item())
    if keep:
        over = (z.double() - want_z).abs() - off_z - 2.0 ** -8 * (want_z.abs() + off_z)
        assert over.max().item() <= 0, over.max().item()
    first = y.clone()
    if not in_place:
        B.qail_w16a16_linear(d, x, y, ws, residual=r, z=z)
        assert torch.equal(first, y)


@pytest.mark.parametrize("M, N, K", [
    (1, 1, 8), (1, 8, 8), (1, 300, 64), (2, 129, 72), (3, 4096, 1024), (16, 257, 4096), (31, 128, 136), (32, 96, 64), (33, 40, 200), (64, 1000, 264),
    (100, 7, 512), (128, 128, 64), (129, 255, 1000), (257, 384, 128), (300, 1, 2048), (289, 1024, 1032), (640, 640, 640), (1, 32000, 256), (1000, 24, 16),
    (513, 769, 320), (2056, 264, 72), (300, 2501, 1000),
    (310, 14905, 520)])
def test_products(B, M, N, K):
    check_forward(B, M, N, K, seed=M + N)


@pytest.mark.parametrize("activation", ACTIVATIONS)
@pytest.mark.parametrize("M, N, K", [(5, 72, 4096), (5, 71, 512), (140, 264, 128), (140, 261, 1024)])
def test_epilogues(B, M, N, K, activation):
    check_forward(B, M, N, K, activation, bias=True, residual=True, keep=True)
    check_forward(B, M, N, K, activation, bias=True, out=torch.float32)
    check_forward(B, M, N, K, activation, residual=True, keep=True, out=torch.float32)
    check_forward(B, M, N, K, activation, bias=True, residual=True, in_place=True)


@pytest.mark.parametrize("M, N", [(5, 71), (140, 261), (33, 9), (200, 7)])
def test_rows_of_an_odd_width_stay_in_their_tensors(B, M, N):
    """Wide stores at any address: what lies behind the last row, and in front of the first, keeps its values."""
    x, w, b, dy = normal((M, 64), 1), normal((N, 64), 2), normal((N,), 3), normal((M, N), 4)
    d = B.make_w16a16(w, b, "silu")
    for dtype in (BF16, torch.float32):
        room = torch.full((M * N + 48,), 7.0, dtype=dtype, device="cuda")
        kept = torch.full((M * N + 48,), 7.0, dtype=BF16, device="cuda")
        B.qail_w16a16_linear(d, x, room[16:16 + M * N].view(M, N), space(B.qail_w16a16_workspace(d, M)), z=kept[16:16 + M * N].view(M, N))
        for t in (room, kept):
            assert (t[:16] == 7).all() and (t[16 + M * N:] == 7).all() and not (t[16:16 + M * N] == 7).all()
    size = B.qail_w16a16_backward_workspace(d, M)
    ws = torch.full((size + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    B.qail_w16a16_backward(d, x, dy, ws[:size], z=kept[16:16 + M * N].view(M, N), dx=torch.empty_like(x), dweight=torch.empty_like(w), dbias=torch.empty(N, device="cuda"))
    assert (ws[size:] == 0x5A).all()


def test_activations_far_out(B):
    """One product of one term: z is exactly what is asked for; the bounds as above."""
    z = torch.cat((torch.linspace(-30, 30, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 100.0, -100.0, 3e4, -3e4, 1e19, -1e19, 3e38, -3e38]))).cuda().to(BF16)
    w = torch.zeros((8, 8), dtype=BF16, device="cuda")
    w[:, 0] = 1
    x = torch.zeros((z.numel(), 8), dtype=BF16, device="cuda")
    x[:, 0] = z
    for activation in ACTIVATIONS:
        d = B.make_w16a16(w, None, activation)
        y = torch.empty((z.numel(), 8), device="cuda")
        ws = space(B.qail_w16a16_workspace(d, z.numel()))
        B.qail_w16a16_linear(d, x, y, ws)
        want, slope = function(activation, z.double())
        assert ((y[:, 3].double() - want).abs() <= 2.0 ** -20 * want.abs() + 2.0 ** -24).all(), activation
        dy, zz, db = torch.ones((z.numel(), 8), device="cuda"), z[:, None].expand(-1, 8).contiguous(), torch.empty(8, device="cuda")
        dx = torch.empty_like(x)
        ws = space(B.qail_w16a16_backward_workspace(d, z.numel()))
        B.qail_w16a16_backward(d, None, dy, ws, z=zz, dx=dx, dbias=db)
        # dx's first column is 8 equal rounded slopes added up
        slope = torch.where(z.double().abs() > 1e10, (z > 0).double() if activation != "none" else torch.ones_like(slope), slope)
        assert ((dx[:, 0].double() - 8 * slope).abs() <= 8 * (2.0 ** -7 * slope.abs() + 2.0 ** -20)).all(), activation
        assert (db.double() - slope.sum()).abs().max().item() <= z.numel() * (2.0 ** -20 * 1.13) + 1e-2, activation


def check_backward(B, M, N, K, activation="none", dtype=BF16, which=("dx", "dweight", "dbias"), seed=0):
    x, w, dy = normal((M, K), seed), normal((N, K), seed + 1, K ** -0.5), normal((M, N), seed + 2, dtype=dtype)
    z = normal((M, N), seed + 3) if activation != "none" else None
    d = B.make_w16a16(w, None, activation)
    nan = lambda shape, t: torch.full(shape, float("nan"), dtype=t, device="cuda")  # noqa: E731
    out = dict(dx=nan((M, K), BF16), dweight=nan((N, K), BF16), dbias=nan((N,), torch.float32))
    out = {k: v for k, v in out.items() if k in which}
    ws = space(B.qail_w16a16_backward_workspace(d, M))
    B.qail_w16a16_backward(d, x if "dweight" in which else None, dy, ws, z=z, **out)
    dz = dy.double() * (function(activation, z.double())[1] if z is not None else 1)
    off_z = 0 if activation in ("none", "relu") else 2.0 ** -20 * dy.double().abs() * z.double().abs().clamp(min=1)
    rounded = 2.0 ** -8 * dz.abs() if not (activation == "none" and dtype == BF16) else torch.zeros_like(dz)
    for name, a, b, R in (("dx", (dz, rounded + off_z), w, N), ("dweight", (dz.t(), (rounded + off_z).t()), x, M)):
        if name in out:
            want = a[0] @ b.double()
            off = (R + 2) * 2.0 ** -23 * (a[0].abs() @ b.double().abs()) * (1 + 2.0 ** -8) + a[1] @ b.double().abs()
            over = (out[name].double() - want).abs() - off - 2.0 ** -8 * (want.abs() + off)
            assert over.max().item() <= 0, (name, over.max().item(), over.argmax().item())
    if "dbias" in out:
        off = (M + 2) * 2.0 ** -23 * dz.abs().sum(0) + (off_z.sum(0) if torch.is_tensor(off_z) else 0)
        over = (out["dbias"].double() - dz.sum(0)).abs() - off
        assert over.max().item() <= 0, ("dbias", over.max().item())
    first = {k: v.clone() for k, v in out.items()}
    B.qail_w16a16_backward(d, x, dy, ws, z=z, **out)
    assert all(torch.equal(first[k], out[k]) for k in out)


@pytest.mark.parametrize("M, N, K", [
    (1, 1, 8), (1, 8, 16), (2, 129, 72), (7, 4096, 256), (32, 96, 64), (33, 41, 200), (64, 1000, 264), (100, 7, 512), (129, 255, 1000), (289, 1024, 136),
    (257, 384, 128), (300, 1, 2048), (640, 640, 640), (1, 2000, 1024), (1100, 24, 16), (65, 130, 8)])
@pytest.mark.parametrize("activation, dtype", [("none", BF16), ("none", torch.float32), ("gelu", BF16)])
def test_gradients(B, M, N, K, activation, dtype):
    check_backward(B, M, N, K, activation, dtype, seed=M + N)


@pytest.mark.parametrize("activation", ACTIVATIONS)
@pytest.mark.parametrize("which", [("dx",), ("dweight",), ("dbias",), ("dx", "dbias"), ("dweight", "dbias"), ("dx", "dweight")])
def test_gradients_one_by_one(B, activation, which):
    check_backward(B, 50, 72, 136, activation, which=which)
    check_backward(B, 70, 75, 136, activation, torch.float32, which=which)


@pytest.mark.parametrize("activation", ACTIVATIONS)
def test_gradients_agree_with_differences(B, activation):
    """Of sum(y * c) in each input, by central differences of the calls themselves with fp32 outputs.  z moves by e = 2^-5 (x, W) of terms of size 1: the
    differences' own error is e^2 / 6 of the third derivative (below 3 each, of the moved terms) and fp32's 2^-22 / e of the sums; dz and z are rounded by 2^-8, the latter
    moving slopes by 1.13 2^-8 |z|."""
    M, N, K = 3, 8, 16
    x, w, b, c = normal((M, K), 1), normal((N, K), 2, 0.25), normal((N,), 3), normal((M, N), 4)
    # no z within reach of relu's corner: it moves by at most e |w| or e |x|
    d = B.make_w16a16(w, b, activation)
    y, z = torch.empty((M, N), device="cuda"), torch.empty((M, N), dtype=BF16, device="cuda")
    B.qail_w16a16_linear(d, x, y, space(B.qail_w16a16_workspace(d, M)), z=z)
    out = dict(dx=torch.empty_like(x), dweight=torch.empty_like(w), dbias=torch.empty(N, device="cuda"))
    B.qail_w16a16_backward(d, x, c, space(B.qail_w16a16_backward_workspace(d, M)), z=z, **out)

    def loss(x, w, b):
        d = B.make_w16a16(w, b, activation)
        y = torch.empty((M, N), device="cuda")
        B.qail_w16a16_linear(d, x, y, space(B.qail_w16a16_workspace(d, M)))
        return (y.double() * c.double()).sum().item()

    zd, cd = (x.double() @ w.double().t() + b.double()), c.double()
    for name, t, at, terms in (("dx", x, (1, 5), w.double()[:, 5] * cd[1]), ("dweight", w, (3, 7), x.double()[:, 7] * cd[:, 3]), ("dbias", b, (2,), cd[:, 2])):
        near = zd[1] if name == "dx" else zd[:, 3] if name == "dweight" else zd[:, 2]
        moved = {"dx": w.double()[:, 5], "dweight": x.double()[:, 7], "dbias": torch.ones(M, device="cuda").double()}[name]
        e = 2.0 ** -5
        up, down = t.clone(), t.clone()
        up[at] += e
        down[at] -= e
        step = (up[at].double() - down[at].double()).item()
        args = lambda v: {"dx": (v, w, b), "dweight": (x, v, b), "dbias": (x, w, v)}[name]  # noqa: E731
        got = (loss(*args(up)) - loss(*args(down))) / step
        size = terms.abs().sum().item()
        off = size * (2.0 ** -7 + 1.13 * 2.0 ** -8 * near.abs().max().item() + 2.0 * (step * moved.abs().max().item()) ** 2) + 2.0 ** -18 / step + 2.0 ** -8 * abs(got)
        if activation == "relu":    # a term whose z changes its sign is off by all of itself
            off += (terms.abs() * (near.abs() <= step * moved.abs())).sum().item()
        assert abs(out[name][at].double().item() - got) <= off, (name, out[name][at].item(), got, off)
