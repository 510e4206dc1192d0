"""The serving operators without a GPU: refusals of the C ABI and of the binding, workspace sizes, and the index arithmetic of the
kernels over bad arrays."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from tests.helpers import ensure_built

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
OK, ODD = 0x10000, 0x10008   # addresses that are never looked at


@pytest.fixture(scope="module")
def B():
    return ensure_built()


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_index_arithmetic_of_the_cache_on_the_host(tmp_path):
    exe = str(tmp_path / "host_cache_driver")
    r = subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-host-only", "-Wno-unused-command-line-argument", "-Xarch_host", "-fsanitize=undefined",
                        "-Xarch_host", "-fno-sanitize-recover=undefined", "-fno-gpu-sanitize",
                        "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2412_01034_amd", "csrc"),
                        os.path.join(ROOT, "tests", "host_cache_driver.cpp"), "-o", exe],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-4000:]
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and "cache: ok" in r.stdout, r.stdout[-4000:]


# ------------------------------------------------------------------------------------------- norm --

def norm(B, **change):
    a = dict(x=OK, residual=None, weight=OK, eps=1e-5, M=4, K=64, h_out=None, y=OK, y_s8=None, y_scale=None)
    a.update(change)
    return B.lib().qail_rmsnorm(*a.values(), None)


def test_rmsnorm_refusals(B):
    for bad in (dict(M=0), dict(M=-1), dict(K=0), dict(K=4), dict(K=60), dict(eps=0.0), dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(residual=OK, h_out=0x20000, y=0x20000)):
        assert norm(B, **bad) == B.QAIL_ERR_SHAPE, bad
    for bad in (dict(K=32776), dict(M=1 << 20, K=4096)):
        assert norm(B, **bad) == B.QAIL_ERR_UNSUPPORTED, bad
    for bad in (dict(x=None), dict(weight=None), dict(y=None), dict(y_s8=OK), dict(y_scale=OK), dict(y=None, h_out=OK)):
        assert norm(B, **bad) == B.QAIL_ERR_NULL, bad
    for bad in (dict(x=ODD), dict(weight=ODD), dict(y=ODD), dict(residual=ODD), dict(residual=OK, h_out=ODD), dict(y_s8=ODD, y_scale=OK), dict(y_s8=OK, y_scale=OK + 2)):
        assert norm(B, **bad) == B.QAIL_ERR_ALIGN, bad


def test_rmsnorm_backward_refusals(B):
    n = B.qail_rmsnorm_backward_workspace(4, 64)
    assert n >= 4 * 64 * 4

    def call(**change):
        a = dict(h=OK, weight=OK, eps=1e-5, dy=OK, dres=None, M=4, K=64, dx=OK, dweight=OK, ws=OK, n=n)
        a.update(change)
        return B.lib().qail_rmsnorm_backward(*a.values(), None)

    for bad in (dict(M=0), dict(K=12), dict(eps=0.0)):
        assert call(**bad) == B.QAIL_ERR_SHAPE, bad
    assert call(K=32776) == B.QAIL_ERR_UNSUPPORTED
    for name in ("h", "weight", "dy", "dx", "dweight"):
        assert call(**{name: None}) == B.QAIL_ERR_NULL, name
        assert call(**{name: ODD}) == B.QAIL_ERR_ALIGN, name
    assert call(dres=ODD) == B.QAIL_ERR_ALIGN and call(ws=ODD) == B.QAIL_ERR_ALIGN
    assert call(ws=None) == B.QAIL_ERR_WORKSPACE and call(n=n - 1) == B.QAIL_ERR_WORKSPACE
    for bad in ((0, 64), (4, 60)):
        with pytest.raises(B.QailError) as e:
            B.qail_rmsnorm_backward_workspace(*bad)
        assert e.value.status == B.QAIL_ERR_SHAPE
    assert B.qail_rmsnorm_backward_workspace(10 ** 6, 2048) == B.qail_rmsnorm_backward_workspace(1000, 2048)   # one row of fp32 a block


# ------------------------------------------------------------------------------- cache and attention --

def cache(B, **change):
    a = dict(k=OK, v=OK, k_scale=None, v_scale=None, num_pages=10, heads=2, page_size=64, head_dim=128, type=B.QAIL_KV_BF16)
    a.update(change)
    return B.qail_kv_cache(*a.values())


def requests(B, **change):
    a = dict(page_table=OK, q_start=OK, kv_len=OK, requests=3, max_pages=5, tokens=7, max_new=4, max_len=320)
    a.update(change)
    return B.qail_requests(*a.values())


BAD_CACHES = [
    (dict(num_pages=0), "SHAPE"), (dict(heads=0), "SHAPE"), (dict(page_size=8), "SHAPE"), (dict(page_size=48), "SHAPE"), (dict(page_size=-64), "SHAPE"),
    (dict(head_dim=0), "SHAPE"), (dict(head_dim=96), "UNSUPPORTED"), (dict(head_dim=256), "UNSUPPORTED"), (dict(page_size=2048), "UNSUPPORTED"),
    (dict(type=2), "UNSUPPORTED"), (dict(type=-1), "UNSUPPORTED"), (dict(heads=1 << 20), "UNSUPPORTED"),
]
BAD_STEPS = [
    (dict(k=None), {}, "NULL"), (dict(v=None), {}, "NULL"), (dict(type=1), {}, "NULL"), (dict(type=1, k_scale=OK), {}, "NULL"),
    (dict(k=ODD), {}, "ALIGN"), (dict(v=ODD), {}, "ALIGN"), (dict(type=1, k_scale=OK, v_scale=ODD), {}, "ALIGN"),
    ({}, dict(requests=0), "SHAPE"), ({}, dict(max_pages=0), "SHAPE"), ({}, dict(tokens=-1), "SHAPE"), ({}, dict(max_new=-1), "SHAPE"),
    ({}, dict(max_len=-1), "SHAPE"), ({}, dict(page_table=None), "NULL"), ({}, dict(q_start=None), "NULL"), ({}, dict(kv_len=None), "NULL"),
    ({}, dict(page_table=OK + 2), "ALIGN"), ({}, dict(q_start=OK + 1), "ALIGN"), ({}, dict(kv_len=OK + 2), "ALIGN"),
    ({}, dict(max_pages=1 << 25), "UNSUPPORTED"), ({}, dict(tokens=1 << 27), "UNSUPPORTED"), ({}, dict(requests=1 << 21), "UNSUPPORTED"),
]


def append(B, c, b, **change):
    a = dict(k=OK, ks=256, v=OK, vs=256, q=OK, qs=512, heads=4, out=0x20000, cos=OK, sin=OK, positions=400, errors=None)
    a.update(change)
    return B.lib().qail_kv_append(ctypes.byref(c), ctypes.byref(b), *a.values(), None)


def attend(B, c, b, **change):
    a = dict(q=OK, qs=512, heads=4, scale=0.1, out=OK, errors=None, ws=OK, n=1 << 30)
    a.update(change)
    return B.lib().qail_paged_attention(ctypes.byref(c), ctypes.byref(b), *a.values(), None)


def test_cache_and_step_refusals(B):
    L = B.lib()
    assert L.qail_kv_cache_sizes(None, None, None) == B.QAIL_ERR_NULL
    for bad, name in BAD_CACHES:
        want = getattr(B, "QAIL_ERR_" + name)
        c = cache(B, **bad)
        assert L.qail_kv_cache_sizes(ctypes.byref(c), None, None) == want, bad
        assert append(B, c, requests(B)) == want and attend(B, c, requests(B)) == want, bad
    n = ctypes.c_size_t()
    for c, b, name in BAD_STEPS:
        want = getattr(B, "QAIL_ERR_" + name)
        assert append(B, cache(B, **c), requests(B, **b)) == want, (c, b)
        assert attend(B, cache(B, **c), requests(B, **b)) == want, (c, b)
        assert L.qail_paged_attention_workspace(ctypes.byref(cache(B, **c)), ctypes.byref(requests(B, **b)), 4, ctypes.byref(n)) == want, (c, b)
    assert L.qail_kv_append(None, ctypes.byref(requests(B)), OK, 256, OK, 256, None, 0, 0, None, None, None, 0, None, None) == B.QAIL_ERR_NULL
    assert L.qail_kv_append(ctypes.byref(cache(B)), None, OK, 256, OK, 256, None, 0, 0, None, None, None, 0, None, None) == B.QAIL_ERR_NULL
    assert L.qail_paged_attention(None, None, OK, 512, 4, 0.1, OK, None, None, 0, None) == B.QAIL_ERR_NULL
    assert L.qail_paged_attention_workspace(ctypes.byref(cache(B)), ctypes.byref(requests(B)), 4, None) == B.QAIL_ERR_NULL
    assert B.qail_kv_cache_sizes(10, 2, 64, 128, B.QAIL_KV_BF16) == (10 * 2 * 64 * 256, 0)
    assert B.qail_kv_cache_sizes(1 << 20, 8, 256, 64, B.QAIL_KV_S8) == ((1 << 31) * 64, (1 << 31) * 4)


def test_kv_append_refusals(B):
    c, b = cache(B), requests(B)
    for bad in (dict(ks=255), dict(ks=248), dict(vs=8), dict(qs=504), dict(qs=513), dict(heads=0), dict(positions=0), dict(q=OK, out=OK, qs=520)):
        assert append(B, c, b, **bad) == B.QAIL_ERR_SHAPE, bad
    for bad in (dict(k=None), dict(v=None), dict(q=None), dict(out=None), dict(cos=None), dict(sin=None), dict(cos=None, sin=None)):
        assert append(B, c, b, **bad) == B.QAIL_ERR_NULL, bad
    for bad in (dict(k=ODD), dict(v=ODD), dict(q=ODD), dict(out=ODD), dict(cos=ODD), dict(sin=ODD), dict(errors=OK + 1)):
        assert append(B, c, b, **bad) == B.QAIL_ERR_ALIGN, bad
    for bad in (dict(ks=1 << 40), dict(heads=1 << 17, qs=1 << 30)):
        assert append(B, c, b, **bad) == B.QAIL_ERR_UNSUPPORTED, bad
    assert append(B, c, requests(B, tokens=0)) == B.QAIL_OK       # nothing to do


def test_paged_attention_refusals(B):
    c, b = cache(B), requests(B)
    need = B.qail_paged_attention_workspace(c, requests(B, requests=1, max_pages=100, max_len=6400), 4)
    assert need > 0 and need % 256 == 0
    for bad in (dict(heads=0), dict(heads=3), dict(heads=-2), dict(qs=504), dict(qs=516), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf"))):
        assert attend(B, c, b, **bad) == B.QAIL_ERR_SHAPE, bad
    for bad in (dict(q=None), dict(out=None)):
        assert attend(B, c, b, **bad) == B.QAIL_ERR_NULL, bad
    for bad in (dict(q=ODD), dict(out=ODD), dict(errors=OK + 2)):
        assert attend(B, c, b, **bad) == B.QAIL_ERR_ALIGN, bad
    long = requests(B, requests=1, max_pages=100, max_len=6400)
    assert attend(B, c, long, ws=None) == B.QAIL_ERR_WORKSPACE and attend(B, c, long, n=need - 1) == B.QAIL_ERR_WORKSPACE
    assert attend(B, c, long, ws=OK + 16, n=need) == B.QAIL_ERR_ALIGN
    assert attend(B, c, requests(B, tokens=1 << 26, max_new=1 << 26), heads=64, qs=8192) == B.QAIL_ERR_UNSUPPORTED
    assert attend(B, c, requests(B, tokens=0)) == B.QAIL_OK
    assert B.qail_paged_attention_workspace(c, requests(B, tokens=0), 4) == 0


def test_sizes_whose_launches_would_be_too_large_are_refused(B):
    """A launch has less than 2^32 threads: rows of a norm have 64 at least, tokens and (request, head) pairs 256."""
    assert norm(B, M=1 << 26, K=8) == B.QAIL_ERR_UNSUPPORTED
    c, many = cache(B), requests(B, tokens=1 << 24)
    assert append(B, c, many, q=None, out=None) == B.QAIL_ERR_UNSUPPORTED and attend(B, c, many) == B.QAIL_ERR_UNSUPPORTED
    heads = (1 << 22) // (1 << 20) + 1
    wide = dict(heads=heads, qs=heads * 128)
    assert attend(B, cache(B, heads=heads), requests(B, requests=1 << 20), **wide) == B.QAIL_ERR_UNSUPPORTED


def test_binding_refuses_what_is_no_device_tensor(B):
    bf = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        B.qail_rmsnorm(bf, bf[0], 1e-5, y=bf)
    with pytest.raises(ValueError, match="bfloat16"):
        B.qail_rmsnorm(bf.float(), bf[0], 1e-5, y=bf)
    k = torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        B.make_kv_cache(k, k)
    with pytest.raises(ValueError, match="one shape"):
        B.make_kv_cache(k, k[:1])
    with pytest.raises(ValueError, match="int8 cache"):
        B.make_kv_cache(k, k, torch.zeros((2, 1, 16)), torch.zeros((2, 1, 16)))
    with pytest.raises(ValueError, match="int8 cache"):
        B.make_kv_cache(k.to(torch.int8), k.to(torch.int8))
    with pytest.raises(ValueError, match="int32"):
        B.make_requests(torch.zeros((1, 1), dtype=torch.int64), torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 1, 1, 1)
    with pytest.raises(ValueError, match="given"):
        B.make_adapters([dict(N=8, K=64, A=torch.zeros((1, 8, 64), dtype=torch.bfloat16), B=torch.zeros((1, 9, 8), dtype=torch.bfloat16),
                              scaling=torch.ones(1))])


# ----------------------------------------------------------------------------------------- adapters --

def test_adapters_refusals(B):
    L = B.lib()

    def lists(r=8, n=2, item=None, adapter=None):
        items, ad = (B.qail_w4a16_item * 1)(), (B.qail_adapters * 1)()
        items[0] = B.qail_w4a16_item(B.qail_wdesc(64, 128, 64, B.QAIL_W4_ASYM_GROUP), OK, OK, OK, OK, OK)
        ad[0] = B.qail_adapters(OK, OK, OK, n, r)
        for name, value in (item or {}).items():
            setattr(items[0], name, value)
        for name, value in (adapter or {}).items():
            setattr(ad[0], name, value)
        return items, ad

    def call(items, ad, rows=OK, count=1, M=3, ws=OK, n=1 << 30):
        return L.qail_w4a16_linear_adapters_batch(items, ad, rows, count, M, ws, n, None)

    need = B.qail_w4a16_adapters_workspace(*lists(), 1, 3)
    assert need >= 3 * 8 * 4
    for bad in (dict(r=0), dict(r=4), dict(r=12), dict(r=72), dict(n=0), dict(n=-1)):
        assert call(*lists(**bad)) == B.QAIL_ERR_SHAPE, bad
    assert call(*lists(), count=-1) == B.QAIL_ERR_SHAPE and call(*lists(), M=0) == B.QAIL_ERR_SHAPE
    assert call(*lists(item=dict(d=B.qail_wdesc(64, 100, 64, 0)))) == B.QAIL_ERR_SHAPE
    assert call(*lists(item=dict(d=B.qail_wdesc(64, 128, 64, B.QAIL_W8_SYM_GROUP)))) == B.QAIL_ERR_UNSUPPORTED
    assert call(*lists(item=dict(d=B.qail_wdesc(1 << 26, 128, 64, 0))), M=64) == B.QAIL_ERR_UNSUPPORTED
    for name in ("qweight", "scales", "zeros", "x", "y"):
        assert call(*lists(item={name: None})) == B.QAIL_ERR_NULL and call(*lists(item={name: ODD})) == B.QAIL_ERR_ALIGN, name
    for name in ("A", "B", "scaling"):
        assert call(*lists(adapter={name: None})) == B.QAIL_ERR_NULL and call(*lists(adapter={name: ODD})) == B.QAIL_ERR_ALIGN, name
    items, ad = lists()
    assert call(None, ad) == B.QAIL_ERR_NULL and call(items, None) == B.QAIL_ERR_NULL and call(items, ad, rows=None) == B.QAIL_ERR_NULL
    assert call(items, ad, rows=OK + 2) == B.QAIL_ERR_ALIGN and call(items, ad, ws=OK + 16) == B.QAIL_ERR_ALIGN
    assert call(items, ad, ws=None) == B.QAIL_ERR_WORKSPACE and call(items, ad, n=need - 1) == B.QAIL_ERR_WORKSPACE
    assert call(items, ad, count=0) == B.QAIL_OK
    assert L.qail_w4a16_adapters_workspace(items, ad, 1, 3, None) == B.QAIL_ERR_NULL


# -------------------------------------------------------------------------------------- marshalling --

def test_native_calls_leave_what_is_not_plain_to_python(B):
    """None for what the compiled marshalling does not take (here: nothing is on a GPU), the library's own errors in Python's words."""
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros(64, dtype=torch.bfloat16)
    assert B._rmsnorm_native(x, w, 1e-5, None, None, x, None, None) is None
    assert B._rmsnorm_backward_native(x, w, 1e-5, x, x, w, x, None) is None
    c, b = cache(B), requests(B)
    t = torch.zeros((7, 2, 128), dtype=torch.bfloat16)
    assert B._kv_append_native(c, b, t, t, None, None, None, None, None) is None
    assert B._paged_attention_native(c, b, t, t, 0.1, None, None) is None
    assert B._adapters_batch_native((B.qail_w4a16_item * 1)(), (B.qail_adapters * 1)(), torch.zeros(1, dtype=torch.int32), 1, 1, x) is None
    for call in (B._rmsnorm_native, B._rmsnorm_backward_native, B._kv_append_native, B._paged_attention_native, B._adapters_batch_native):
        assert call() is None and call(*[None] * 8) is None and call(*[5] * 7) is None
    # structures of other kinds, also of the same size, are none of the cache's
    item = B.qail_w4a16_item()
    assert ctypes.sizeof(item) == ctypes.sizeof(c)
    with pytest.raises((ctypes.ArgumentError, AttributeError)):
        B.qail_paged_attention(item, b, t, t, 0.1)
    with pytest.raises((ctypes.ArgumentError, ValueError)):
        B.qail_w4a16_linear_adapters_batch((B.qail_adapters * 1)(), (B.qail_adapters * 1)(), torch.zeros(1, dtype=torch.int32), 1, 1, x)
