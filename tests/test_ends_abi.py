"""The policy's 16-bit ends without a GPU: refusals of the C ABI and of the binding, workspace sizes, and how products are divided."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from tests.helpers import ROOT, ensure_built

HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
OK, ODD = 0x10000, 0x10008   # addresses that are never looked at
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def B():
    return ensure_built()


def expect(status, call, *changes):
    for c in changes:
        assert call(**c) == status, c


def test_embed_refusals(B):
    def call(**change):
        a = dict(table=OK, V=100, K=64, ids=OK, T=5, scale=1.0, h=0x20000, errors=None)
        a.update(change)
        return B.lib().qail_embed(*a.values(), None)

    expect(B.QAIL_ERR_SHAPE, call, dict(V=0), dict(K=0), dict(K=4), dict(K=60), dict(T=-1), dict(scale=NAN), dict(scale=INF), dict(scale=-INF), dict(h=OK))
    expect(B.QAIL_ERR_UNSUPPORTED, call, dict(K=65544), dict(V=1 << 24), dict(T=1 << 24), dict(V=(1 << 24) - 1, K=8192), dict(T=(1 << 24) - 1, K=8192))
    expect(B.QAIL_ERR_NULL, call, dict(table=None), dict(ids=None), dict(h=None))
    expect(B.QAIL_ERR_ALIGN, call, dict(table=ODD), dict(ids=OK + 2), dict(h=ODD), dict(errors=OK + 2))
    expect(B.QAIL_OK, call, dict(T=0), dict(T=0, ids=None, h=None))


def test_embed_backward_refusals(B):
    n = B.qail_embed_backward_workspace(100, 64, 5000)

    def call(**change):
        a = dict(ids=OK, dh=OK, T=5000, scale=1.0, V=100, K=64, accumulate=0, dtable=OK + 4096, errors=None, ws=OK, bytes=n)
        a.update(change)
        return B.lib().qail_embed_backward(*a.values(), None)

    expect(B.QAIL_ERR_SHAPE, call, dict(V=0), dict(K=12), dict(T=-1), dict(scale=NAN), dict(dtable=OK))
    expect(B.QAIL_ERR_UNSUPPORTED, call, dict(K=65544), dict(V=1 << 24), dict(T=1 << 24))
    expect(B.QAIL_ERR_NULL, call, dict(ids=None), dict(dh=None), dict(dtable=None))
    expect(B.QAIL_ERR_ALIGN, call, dict(ids=OK + 2), dict(dh=ODD), dict(dtable=ODD), dict(ws=OK + 16), dict(errors=OK + 1))
    expect(B.QAIL_ERR_WORKSPACE, call, dict(ws=None), dict(bytes=n - 1))
    expect(B.QAIL_OK, call, dict(T=0, accumulate=1, ws=None, bytes=0))
    assert n >= 4 * 5000 * 4                      # keys and places, twice
    with pytest.raises(B.QailError):
        B.qail_embed_backward_workspace(100, 63, 5)


def linear(B, **change):
    a = dict(N=96, K=64, activation=B.QAIL_ACT_GELU, weight=OK, bias=None)
    a.update(change)
    return B.qail_w16a16(*a.values())


def test_linear_refusals(B):
    def call(d={}, none=False, **change):
        a = dict(x=OK, M=4, residual=None, z=None, y=0x20000, y32=None, ws=OK, bytes=1 << 30)
        a.update(change)
        return B.lib().qail_w16a16_linear(None if none else ctypes.byref(linear(B, **d)), *a.values(), None)

    expect(B.QAIL_ERR_SHAPE, call, dict(M=0), dict(M=-1), dict(d=dict(N=0)), dict(d=dict(K=0)), dict(d=dict(K=60)), dict(y=OK), dict(z=0x20000),
           dict(z=0x30000, residual=0x30000), dict(z=OK), dict(y=None, y32=0x30000, residual=0x30000), dict(y=None, y32=OK), dict(y=None, y32=0x30000, z=0x30000))
    expect(B.QAIL_ERR_UNSUPPORTED, call, dict(d=dict(activation=5)), dict(d=dict(activation=-1)), dict(M=(1 << 22) + 1), dict(d=dict(N=(1 << 22) + 8)),
           dict(d=dict(K=(1 << 22) + 8)), dict(M=1 << 22, d=dict(N=4096)), dict(M=1 << 22, d=dict(K=4096)), dict(d=dict(N=1 << 20, K=1 << 14)))
    expect(B.QAIL_ERR_NULL, call, dict(none=True), dict(x=None), dict(y=None), dict(y32=OK), dict(d=dict(weight=None)))
    expect(B.QAIL_ERR_ALIGN, call, dict(x=ODD), dict(y=0x20008), dict(y=None, y32=ODD), dict(residual=ODD), dict(z=ODD), dict(d=dict(weight=ODD)), dict(d=dict(bias=ODD)))
    big = dict(N=4096, K=4096)                    # few tiles: K is divided
    assert call(d=big, y=0x30000, residual=0x30000, ws=None) == B.QAIL_ERR_WORKSPACE    # in place: gets past the pointers
    n = B.qail_w16a16_workspace(linear(B, **big), 4)
    assert n >= 2 * 4 * 4096 * 4
    expect(B.QAIL_ERR_WORKSPACE, call, dict(d=big, ws=None), dict(d=big, bytes=n - 1))
    expect(B.QAIL_ERR_ALIGN, call, dict(d=big, ws=OK + 16))


def test_an_output_in_place_of_the_residual_is_no_other_input(B):
    """x + f(x) in place would have blocks read rows of x that others have overwritten.  (Sizes that need a workspace, which is missing: no call gets as far as a launch.)"""
    def call(d={}, **change):
        a = dict(x=OK, M=4, residual=0x30000, z=None, y=0x30000, y32=None, ws=None, bytes=0)
        a.update(change)
        d = dict(dict(N=4096, K=4096, weight=0x50000, bias=0x60000), **d)
        return B.lib().qail_w16a16_linear(ctypes.byref(linear(B, **d)), *a.values(), None)

    expect(B.QAIL_ERR_WORKSPACE, call, dict())
    expect(B.QAIL_ERR_SHAPE, call, dict(x=0x30000), dict(d=dict(weight=0x30000)), dict(d=dict(bias=0x30000)), dict(z=0x30000), dict(z=OK), dict(z=0x50000), dict(z=0x60000),
           dict(y=None, y32=0x30000), dict(y=None, y32=0x60000), dict(y=None, y32=0x70000, z=0x30000))


def test_linear_backward_refusals(B):
    n = B.qail_w16a16_backward_workspace(linear(B), 4)

    def call(d={}, **change):
        a = dict(x=OK, z=OK, dy=OK, dy32=None, M=4, dx=0x20000, dweight=0x30000, dbias=0x40000, ws=OK, bytes=n)
        a.update(change)
        return B.lib().qail_w16a16_backward(ctypes.byref(linear(B, **d)), *a.values(), None)

    expect(B.QAIL_ERR_SHAPE, call, dict(M=0), dict(d=dict(K=4)), dict(dx=OK), dict(dweight=OK), dict(dbias=OK), dict(dx=0x30000), dict(dbias=0x20000))
    expect(B.QAIL_ERR_UNSUPPORTED, call, dict(d=dict(activation=9)), dict(M=1 << 23))
    expect(B.QAIL_ERR_NULL, call, dict(x=None), dict(z=None), dict(dy=None), dict(dy32=OK), dict(dx=None, dweight=None, dbias=None), dict(d=dict(weight=None)))
    expect(B.QAIL_ERR_ALIGN, call, dict(x=ODD), dict(z=ODD), dict(dy=ODD), dict(dy=None, dy32=ODD), dict(dx=0x20008), dict(dweight=0x30008), dict(dbias=0x40008),
           dict(ws=OK + 16), dict(d=dict(weight=ODD)))
    expect(B.QAIL_ERR_WORKSPACE, call, dict(ws=None), dict(bytes=n - 1))


def test_sample_refusals(B):
    def call(s={}, none=False, **change):
        a = dict(logits=OK, type=B.QAIL_LOGITS_F32, stride=1000, R=4, V=1000)
        b = dict(u=OK, token=OK, logprob=None, errors=None)
        a.update({k: v for k, v in change.items() if k in a})
        b.update({k: v for k, v in change.items() if k in b})
        c = B.qail_sampling(**s)
        return B.lib().qail_sample(*a.values(), None if none else ctypes.byref(c), *b.values(), None)

    expect(B.QAIL_ERR_SHAPE, call, dict(R=-1), dict(V=0), dict(stride=999), dict(stride=-1000))
    expect(B.QAIL_ERR_UNSUPPORTED, call, dict(type=2), dict(type=-1), dict(R=(1 << 20) + 1), dict(V=(1 << 18) + 1, stride=1 << 20), dict(stride=1 << 37))
    expect(B.QAIL_ERR_NULL, call, dict(logits=None), dict(u=None), dict(token=None), dict(none=True))
    expect(B.QAIL_ERR_ALIGN, call, dict(logits=ODD), dict(u=OK + 2), dict(token=OK + 1), dict(logprob=OK + 2), dict(errors=OK + 2), dict(s=dict(temperature=OK + 2)),
           dict(s=dict(top_k=OK + 1)), dict(s=dict(top_p=OK + 2)), dict(s=dict(min_p=OK + 2)))
    expect(B.QAIL_OK, call, dict(R=0), dict(R=0, logits=None, u=None, token=None))


def test_the_binding_refuses_what_is_not_what_it_says(B):
    half, whole, number = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((4, 64)), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor expected"):
        B.qail_embed(half, number, half.clone())
    with pytest.raises(ValueError, match="table: bfloat16"):
        B.qail_embed(whole, number, half)
    with pytest.raises(ValueError, match="ids: int32"):
        B.qail_embed_backward(number.long(), half, whole, half)
    with pytest.raises(ValueError, match="activation: one of"):
        B.make_w16a16(half, activation="tanh")
    with pytest.raises(ValueError, match="weight: bfloat16"):
        B.make_w16a16(whole)
    with pytest.raises(ValueError, match="logits: bfloat16 or float32"):
        B.qail_sample(half.half(), torch.zeros(4), number)
    with pytest.raises(ValueError, match="device tensor expected"):
        B.qail_sample(whole, torch.zeros(4), number)


def test_the_binding_counts_rows_by_the_last_dimension(B):
    new = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)  # noqa: E731
    d, one = B.qail_w16a16(40, 64, 0, OK, None), B.qail_w16a16(1, 64, 0, OK, None)
    for x in (new(4, 128), new(64, 4), new(4), new(4, 64, 1), new(256)):
        with pytest.raises(ValueError, match="x: rows of 64 values expected"):
            B.qail_w16a16_linear(d, x, new(256, 40))
    for dy in (new(4, 80), new(40, 4), new(5)):
        with pytest.raises(ValueError, match="dy: rows of 40 values expected"):
            B.qail_w16a16_backward(d, None, dy, None, dx=new(256, 64))
    with pytest.raises(ValueError, match="dy: rows of 1 values expected"):
        B.qail_w16a16_backward(one, None, new(3, 5), None, dx=new(256, 64))
    for t, n, rows in ((new(3, 5, 64), 64, 15), (new(64), 64, 1), (new(7), 1, 7), (new(7, 1), 1, 7), (new(1), 1, 1), (new(0, 64), 64, 0), (new(2, 0, 64), 64, 0)):
        assert B._rows(t, n, "x") == rows
    with pytest.raises(ValueError, match="y: 1120 bytes given, 1200 needed"):     # 15 rows, not 3
        B.qail_w16a16_linear(d, new(3, 5, 64), new(14, 40))


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_division_of_products_on_the_host(tmp_path):
    exe = str(tmp_path / "host_products_driver")
    r = subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-host-only", "-Wno-unused-command-line-argument", "-Xarch_host", "-fsanitize=undefined",
                        "-Xarch_host", "-fno-sanitize-recover=undefined", "-fno-gpu-sanitize",
                        "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2412_01034_amd", "csrc"),
                        os.path.join(ROOT, "tests", "host_products_driver.cpp"), "-o", exe],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-4000:]
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and "products: ok" in r.stdout, r.stdout[-4000:]
