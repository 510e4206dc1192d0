"""GPU parity of the serving operators against plain forms in 64 bits.  Every tolerance counts roundings: half a step is
2^-8 of a bf16 value and 2^-24 of an fp32 one; codes are decided in fp32 with one rounding an operation and have to be equal."""
import math

import pytest
import torch

from tests import serve_reference as P
from tests.helpers import ensure_built

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    return ensure_built()


def within(got, want, tol, what=""):
    off = (got.double().cpu() - want).abs()
    assert bool(torch.isfinite(got.float()).all()), what
    over = (off - tol).max().item()
    assert over <= 0, (what, "over by %g at %g" % (over, want.flatten()[(off - tol).flatten().argmax()].item()))


# ------------------------------------------------------------------------------------------- norm --

# one thread group of each kind, rows that end inside a group's last piece, the widest row, one value of eight
WIDTHS = [8, 136, 512, 520, 1024, 2048, 2056, 4096, 5120, 8192, 8200, 16384, 16392, 32768]


def norm_inputs(M, K, seed, residual):
    x = P.normal((M, K), seed).to(BF16)
    x[:, ::max(1, K // 3)] *= 10
    if M > 1:
        x[1] = 0
    return x, P.normal((M, K), seed + 1).to(BF16) if residual else None, (1 + P.normal((K,), seed + 2, 0.2)).to(BF16)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,K", [(3, k) for k in WIDTHS] + [(1, 4096), (257, 264), (130, 4096)])
def test_rmsnorm(B, M, K, residual):
    eps = 1e-5
    x, res, w = norm_inputs(M, K, 100 + K, residual)
    xd, wd, rd = x.cuda(), w.cuda(), res.cuda() if residual else None
    h = torch.full((M, K), math.nan, dtype=BF16, device="cuda") if residual else None
    y = torch.full((M, K), math.nan, dtype=BF16, device="cuda")
    codes = torch.full((M, K), 77, dtype=torch.int8, device="cuda")
    scale = torch.full((M,), math.nan, device="cuda")
    B.qail_rmsnorm(xd, wd, eps, residual=rd, residual_out=h, y=y, y_s8=codes, y_scale=scale)
    torch.cuda.synchronize()
    h_ref, y_ref, r = P.rmsnorm(x, res, w, eps)
    if residual:
        within(h, h_ref, (2 ** -8 + 2 ** -23) * h_ref.abs(), "h")
    # r: 8 K / 256 sums in a row and a tree, a root and a quotient: below 2^-18
    within(y, y_ref, (2 ** -8 + 2 ** -18) * y_ref.abs() + 1e-38, "y")
    q, step = P.rmsnorm_codes(x, res, w)
    assert torch.equal(codes.cpu(), q)
    want = step.double() * r[:, 0]
    within(scale, want, 2 ** -18 * want, "scale")
    # one output at a time, the same bits; over their inputs where that is allowed
    alone = torch.empty_like(y)
    B.qail_rmsnorm(xd, wd, eps, residual=rd, y=alone)
    assert torch.equal(alone, y)
    over = torch.empty_like(codes), torch.empty_like(scale)
    if residual:
        B.qail_rmsnorm(xd, wd, eps, residual=rd, residual_out=rd, y=xd, y_s8=over[0], y_scale=over[1])
        assert torch.equal(rd, h) and torch.equal(xd, y)
    else:
        B.qail_rmsnorm(xd, wd, eps, y_s8=over[0], y_scale=over[1])
    assert torch.equal(over[0], codes) and torch.equal(over[1], scale)


def test_rmsnorm_codes_are_activations_of_the_8_bit_linear(B):
    """The codes go into qail_w8a8_gemm as they are; its sums times the row's scale and the weight's are the product."""
    M, K, N = 37, 256, 48
    x, _, w = norm_inputs(M, K, 7, False)
    weight = P.normal((N, K), 8, 0.05)
    codes, scale = torch.empty((M, K), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    B.qail_rmsnorm(x.cuda(), w.cuda(), 1e-5, y_s8=codes, y_scale=scale)
    qw, sw = torch.empty((N, K), dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    B.qail_quantize_weights(weight.cuda(), K, B.QAIL_W8_SYM_CHANNEL, qw, sw, None)
    acc = torch.empty((M, N), dtype=torch.int32, device="cuda")
    B.qail_w8a8_gemm(M, 1, 1, K, N, 1, 1, 1, 0, codes, qw, acc_out=acc)
    assert torch.equal(acc.cpu().long(), codes.cpu().long() @ qw.cpu().long().T)
    y = acc.double().cpu() * scale.double().cpu()[:, None] * sw.double().cpu()
    _, ref, _ = P.rmsnorm(x, None, w, 1e-5)
    # half a step of each side's codes per product
    tol = (scale.double().cpu()[:, None] / 2 * weight.double().abs().sum(1)) + (ref.abs() + scale.double().cpu()[:, None] / 2) @ torch.ones(K, N, dtype=P.F64) * sw.double().cpu() / 2
    assert bool(((y - ref @ weight.double().T).abs() <= tol * 1.001).all())


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,K", [(5, k) for k in WIDTHS] + [(1, 4096), (700, 264), (1100, 4096)])   # also more rows than blocks
def test_rmsnorm_backward(B, M, K, residual):
    eps = 1e-5
    h, dres, w = norm_inputs(M, K, 300 + K, residual)
    dy = P.normal((M, K), 301 + K).to(BF16)
    dx = torch.full((M, K), math.nan, dtype=BF16, device="cuda")
    dw = torch.full((K,), math.nan, device="cuda")
    ws = torch.empty(B.qail_rmsnorm_backward_workspace(M, K), dtype=torch.uint8, device="cuda")
    hd, wd, dyd, rd = h.cuda(), w.cuda(), dy.cuda(), dres.cuda() if residual else None
    B.qail_rmsnorm_backward(hd, wd, eps, dyd, dx, dw, ws, dres=rd)
    torch.cuda.synchronize()
    dx_ref, size, dw_ref, dw_size = P.rmsnorm_backward(h, w, eps, dy, dres)
    within(dx, dx_ref, 2 ** -8 * dx_ref.abs() + 2 ** -17 * size + 1e-38, "dx")   # r and the mean: 2^-18 each
    within(dw, dw_ref, 2 ** -17 * dw_size, "dweight")                            # r, and chains of M / 512 + 48 sums
    again = torch.empty_like(dw)
    B.qail_rmsnorm_backward(hd, wd, eps, dyd, dyd, again, ws, dres=rd)           # over an input; a fixed order of summation
    assert torch.equal(again, dw) and torch.equal(dyd, dx)


def test_rmsnorm_backward_against_differences(B):
    """The gradient of sum(c * y) by central differences of the 64-bit formula (truncation: step^2, far below the outputs' rounding)."""
    M, K, eps, step = 4, 64, 1e-5, 1e-5
    h, _, w = norm_inputs(M, K, 900, False)
    h[1] = P.normal((K,), 901).to(BF16)   # (a row of zeros bends within the step)
    c = P.normal((M, K), 902).to(BF16)
    f = lambda hh, ww: (c.double() * hh / torch.sqrt((hh * hh).mean(1, keepdim=True) + eps) * ww).sum()  # noqa: E731
    dh, dw = torch.zeros(M, K, dtype=P.F64), torch.zeros(K, dtype=P.F64)
    for k in range(K):
        d = torch.zeros(K, dtype=P.F64)
        d[k] = step
        dw[k] = (f(h.double(), w.double() + d) - f(h.double(), w.double() - d)) / (2 * step)
        for m in range(M):
            e = torch.zeros(M, K, dtype=P.F64)
            e[m] = d
            dh[m, k] = (f(h.double() + e, w.double()) - f(h.double() - e, w.double())) / (2 * step)
    dx, dweight = torch.empty((M, K), dtype=BF16, device="cuda"), torch.empty(K, device="cuda")
    ws = torch.empty(B.qail_rmsnorm_backward_workspace(M, K), dtype=torch.uint8, device="cuda")
    B.qail_rmsnorm_backward(h.cuda(), w.cuda(), eps, c.cuda(), dx, dweight, ws)
    _, size, _, dw_size = P.rmsnorm_backward(h, w, eps, c, None)
    within(dx, dh, 2 ** -8 * dh.abs() + 2 ** -16 * size + 1e-7, "dx")
    within(dweight, dw, 2 ** -16 * dw_size + 1e-7, "dweight")


# ------------------------------------------------------------------------------------------- append --

APPENDS = [
    # new tokens, lengths, heads, heads of the cache, head_dim, page
    ([1], [1], 1, 1, 64, 16),
    ([1] * 5, [1, 16, 17, 300, 64], 32, 32, 128, 64),
    ([3, 0, 40, 1], [3, 9, 55, 130], 8, 2, 64, 32),
    ([70, 33], [70, 100], 14, 7, 128, 16),
    ([1] * 200, [1 + 3 * i % 90 for i in range(200)], 4, 1, 128, 1024),   # more requests than a wave has lanes
]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page", APPENDS)
def test_kv_append(B, new, lens, heads, kv_heads, dim, page, eight):
    s = P.Step(new, lens, heads, kv_heads, dim, page, eight, 50 + page, pad=24)
    k, v, ks, vs = s.pools("cuda")
    before = [t.clone() if t is not None else None for t in (k, v, ks, vs)]
    cache = B.make_kv_cache(k, v, ks, vs)
    tensors = s.table.cuda(), s.starts.cuda(), s.kv_len.cuda()
    req = B.make_requests(*tensors, tokens=s.tokens, max_new=max(new), max_len=max(lens))
    cos, sin = P.angles(max(lens), dim)
    qkv, errors = s.qkv.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    q, nk, nv = s.split(qkv)
    q_out = torch.full((s.tokens, heads, dim), math.nan, dtype=BF16, device="cuda")
    B.qail_kv_append(cache, req, nk, nv, q=q, q_out=q_out, cos=cos.cuda(), sin=sin.cuda(), errors=errors)
    torch.cuda.synchronize()
    assert errors.item() == 0
    at = P.positions(s)
    p = torch.tensor([i for _, i in at])
    hq, hk, hv = (t.float() for t in s.split(s.qkv))
    c, sn = cos[p][:, None], sin[p][:, None]
    assert torch.equal(q_out.cpu(), P.rotate(hq, c, sn).to(BF16))
    # every slot of the cache: the new tokens' and all others
    for got, scale, was, was_scale, t in ((k, ks, before[0], before[2], P.rotate(hk, c, sn)), (v, vs, before[1], before[3], hv)):
        want, want_scale = was.cpu(), was_scale.cpu() if eight else None
        codes, step = P.codes_of(t)
        for i, (r, pos) in enumerate(at):
            page_id, slot = int(s.table[r, pos // page]), pos % page
            want[page_id, :, slot] = codes[i] if eight else t[i].to(BF16)
            if eight:
                want_scale[page_id, :, slot] = step[i]
        if eight:
            assert torch.equal(got.cpu(), want)
            assert torch.equal(scale.cpu().view(torch.int32), want_scale.view(torch.int32))
        else:
            assert torch.equal(got.cpu().view(torch.int16), want.view(torch.int16))
    # without a rotation, and the queries over themselves
    B.qail_kv_append(cache, req, nk, nv)
    r, pos = at[-1]
    last = k[int(s.table[r, pos // page]), :, pos % page].cpu()
    assert torch.equal(last, P.codes_of(hk[-1])[0] if eight else hk[-1].to(BF16))
    own = q.contiguous()
    B.qail_kv_append(cache, req, nk, nv, q=own, q_out=own, cos=cos.cuda(), sin=sin.cuda())
    assert torch.equal(own, q_out)


def test_kv_append_of_a_zero_head(B):
    """A head of zeros has step 1 and codes 0."""
    s = P.Step([2], [2], 1, 1, 64, 16, True, 3)
    s.qkv.zero_()
    k, v, ks, vs = s.pools("cuda")
    tensors = s.table.cuda(), s.starts.cuda(), s.kv_len.cuda()
    req = B.make_requests(*tensors, tokens=2, max_new=2, max_len=2)
    _, nk, nv = s.split(s.qkv.cuda())
    B.qail_kv_append(B.make_kv_cache(k, v, ks, vs), req, nk, nv)
    page = int(s.table[0, 0])
    assert not k[page, 0, :2].any() and not v[page, 0, :2].any() and bool((ks[page, 0, :2] == 1).all())


# ---------------------------------------------------------------------------------------- attention --

ATTENDS = [
    # one token of one key; lengths around tiles and pages; some requests wait; grouped heads; a chunk behind nothing and behind a history
    ([1], [1], 1, 1, 64, 16),
    ([1] * 6, [1, 31, 32, 33, 127, 129], 4, 4, 128, 16),
    ([1, 0, 1, 1], [700, 5, 64, 2], 8, 1, 64, 64),
    ([1], [3000], 4, 2, 128, 32),                  # the keys are divided among blocks
    ([1] * 3, [2500, 40, 900], 16, 1, 128, 128),   # ... of ragged requests, all rows of a tile used
    ([1, 1], [600, 333], 24, 1, 64, 16),           # more heads share a head of the cache than a tile has rows
    ([5, 2, 16], [5, 90, 300], 2, 2, 128, 16),
    ([40], [40], 2, 1, 64, 32),
    ([130, 64, 1, 0, 33], [130, 500, 77, 10, 1033], 4, 2, 128, 64),
    ([257], [257], 3, 3, 128, 1024),
    ([100, 3], [2100, 1500], 8, 8, 64, 256),
    ([300, 20], [300, 20], 14, 2, 128, 16),        # seven heads to one of the cache
    ([4, 3], [2, 0], 2, 1, 64, 16),                # more new tokens than a length: the first see nothing, or none does
    ([200], [150], 4, 4, 128, 64),
]


def attention(B, s, scale, max_new=None, max_len=None):
    pools = s.pools("cuda")
    keep = s.table.cuda(), s.starts.cuda(), s.kv_len.cuda(), s.qkv.cuda(), pools
    cache = B.make_kv_cache(*pools)
    req = B.make_requests(*keep[:3], tokens=s.tokens, max_new=max(s.new) if max_new is None else max_new,
                          max_len=max(max(s.lens), 0) if max_len is None else max_len)
    errors = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((s.tokens, s.heads, s.dim), math.nan, dtype=BF16, device="cuda")
    n = B.qail_paged_attention_workspace(cache, req, s.heads)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None    # NaN in whatever is read before it is written
    B.qail_paged_attention(cache, req, s.split(keep[3])[0], out, scale, ws, errors=errors)
    torch.cuda.synchronize()
    assert errors.item() == 0
    return out


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page", ATTENDS)
def test_paged_attention(B, new, lens, heads, kv_heads, dim, page, eight):
    s = P.Step(new, lens, heads, kv_heads, dim, page, eight, 1000 + page + sum(lens), pad=8)
    scale = 1 / math.sqrt(dim)
    out = attention(B, s, scale)
    want, tol = P.attend(s, scale)
    within(out, want, tol)
    assert torch.equal(attention(B, s, scale), out)        # the same bits each time
    # bounds that are not met, and bounds that are far away, plan other launches; the results stay
    for max_new, max_len in ((1, 1), (max(new), 10 ** 6)):
        within(attention(B, s, scale, max_new, max_len), want, tol, (max_new, max_len))


@pytest.mark.parametrize("eight", [False, True])
def test_paged_attention_scores_of_any_size(B, eight):
    """Scores of some hundreds (one key takes all) and near zero (all alike), with either sign of the largest."""
    for scale, seed in ((30.0, 1), (1e-6, 2)):
        s = P.Step([3, 50], [200, 90], 2, 1, 64, 16, eight, seed)
        want, tol = P.attend(s, scale)
        within(attention(B, s, scale), want, tol, scale)
    s = P.Step([2], [70], 1, 1, 64, 16, False, 5)
    s.qkv[:, :64] = 1.0
    s.values[0][0] = -s.values[0][0].abs() * 3     # every score far below zero
    want, tol = P.attend(s, 1.0)
    within(attention(B, s, 1.0), want, tol)


# the last keys of the first request, from one on, hold what is not finite: few rows, rows of many tokens, grouped heads, both kernels in one call,
# keys that are divided among blocks
UNSEEN = [([5], [90], 2, 1, 64, 16, 87), ([4, 3], [4, 40], 4, 4, 128, 16, 1), ([70], [70], 2, 1, 128, 16, 33), ([200, 2], [1300, 9], 4, 1, 64, 32, 1250), ([9], [2500], 1, 1, 128, 64, 2495)]


@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page,first", UNSEEN)
def test_what_a_token_does_not_see_stays_out(B, new, lens, heads, kv_heads, dim, page, first, eight, value):
    """An infinity or NaN in a later token's value (one of its values, or its step) and NaN in its key: the rows in front of it are what they are without
    it, the rows that see it are not finite in the values concerned."""
    s = P.Step(new, lens, heads, kv_heads, dim, page, eight, 700 + first, pad=8)
    scale = 1 / math.sqrt(dim)
    want, tol = P.attend(s, scale)
    rows = torch.arange(s.tokens)
    sees = (rows < new[0]) & (lens[0] - new[0] + rows >= first)
    at = slice(None) if eight else 3
    for only_v in (True, False):
        k, v = s.values[0]
        for t in (v,) if only_v else (k, v):
            if eight:
                t[1][:, first] = value if t is v else math.nan
            else:
                t[:, first, 3] = value if t is v else math.nan
        out = attention(B, s, scale)
        within(out[~sees], want[~sees], tol[~sees], "before")
        got = out[sees].float().cpu()
        assert not torch.isfinite(got[..., at] if only_v else got).any()
        if not eight and only_v:
            others = torch.arange(dim) != 3
            within(out[sees][..., others], want[sees][..., others], tol[sees][..., others], "beside")


def test_paged_attention_beyond_32_bits(B):
    """Pages that lie more than 4 GB into the cache."""
    s = P.Step([1, 40], [200, 100], 2, 1, 128, 256, False, 9, pool=70000)    # 70000 pages of 64 KB
    shape = (s.num_pages, 1, 256, 128)
    small = P.Step([1, 40], [200, 100], 2, 1, 128, 256, False, 9)
    k, v = torch.empty(shape, dtype=BF16, device="cuda"), torch.empty(shape, dtype=BF16, device="cuda")
    used = s.table[s.table > 0]
    used = used[used < s.num_pages].tolist()
    assert min(used) * 65536 > 2 ** 32
    sk, sv, _, _ = small.pools("cuda")
    for r in range(2):
        k[int(s.table[r, 0])], v[int(s.table[r, 0])] = sk[int(small.table[r, 0])], sv[int(small.table[r, 0])]
    keep = s.table.cuda(), s.starts.cuda(), s.kv_len.cuda(), s.qkv.cuda()
    cache, req = B.make_kv_cache(k, v), B.make_requests(*keep[:3], tokens=s.tokens, max_new=40, max_len=200)
    out = torch.empty((s.tokens, 2, 128), dtype=BF16, device="cuda")
    n = B.qail_paged_attention_workspace(cache, req, 2)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    q, nk, nv = s.split(keep[3])
    B.qail_paged_attention(cache, req, q, out, 0.1, ws)
    want, tol = P.attend(small, 0.1)
    within(out, want, tol)
    B.qail_kv_append(cache, req, nk, nv)     # ... and are written to
    torch.cuda.synchronize()
    assert torch.equal(k[int(s.table[1, 0]), 0, 99], nk[-1, 0]) and torch.equal(v[int(s.table[0, 0]), 0, 199], nv[0, 0])


def test_bad_arrays_are_counted_and_fault_nothing(B):
    """The kernels' own checks (tests/test_serve_abi.py walks through them on the CPU): bad pages, lengths and starts."""
    def run(change, append):
        s = P.Step([2, 3], [20, 40], 2, 1, 64, 16, False, 21)
        t = [s.table.cuda(), s.starts.cuda(), s.kv_len.cuda()]
        change(*t)
        k, v, _, _ = s.pools("cuda")
        was = k.clone()
        cache, req = B.make_kv_cache(k, v), B.make_requests(*t, tokens=5, max_new=3, max_len=40)
        errors, out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((5, 2, 64), dtype=BF16, device="cuda")
        q, nk, nv = s.split(s.qkv.cuda())
        if append:
            cos, sin = (a.cuda() for a in P.angles(40, 64))
            B.qail_kv_append(cache, req, nk, nv, q=q, q_out=out, cos=cos, sin=sin, errors=errors)
        else:
            n = B.qail_paged_attention_workspace(cache, req, 2)
            ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
            B.qail_paged_attention(cache, req, q, out, 0.125, ws, errors=errors)
        torch.cuda.synchronize()
        return errors.item(), s, k, was

    def page(value):
        return lambda table, starts, lens: table[1].__setitem__(2, value)      # the page of the second request's last tokens

    for value in (-1, 1000, 2 ** 31 - 1, -2 ** 31):
        for append in (False, True):
            count, s, k, was = run(page(value), append)
            assert count > 0
            if append:    # the good request's tokens were written, the bad one's nowhere
                new = (k.view(torch.int16) != was.view(torch.int16)).any(-1).nonzero()
                assert {int(p) for p in new[:, 0]} == {int(s.table[0, 1])}
    for change in (lambda t, s, l: l.__setitem__(0, 10 ** 6), lambda t, s, l: l.__setitem__(1, -5), lambda t, s, l: s.__setitem__(1, 9),
                   lambda t, s, l: s.__setitem__(1, -3), lambda t, s, l: s.__setitem__(2, 1)):
        for append in (False, True):
            assert run(change, append)[0] > 0
    assert run(lambda t, s, l: l.__setitem__(0, 1), True)[0] > 0      # a negative position has no slot


# ------------------------------------------------------------------------------- graphs and streams --

def test_step_in_a_graph_and_on_another_stream(B):
    """Append and attention captured once and replayed as the requests grow; each replay against an eager call on another stream."""
    heads, kv_heads, dim, page, R = 8, 2, 128, 16, 3
    lens = torch.tensor([5, 31, 200])
    pools = [torch.zeros((60, kv_heads, page, dim), dtype=BF16, device="cuda") for _ in range(2)]
    for t in pools:
        t.normal_(generator=torch.Generator(device="cuda").manual_seed(4))
    twin = [t.clone() for t in pools]
    table = torch.randperm(60, generator=P.gen(5))[:R * 16].view(R, 16).to(torch.int32).cuda()
    starts, kv_len = torch.arange(R + 1, dtype=torch.int32, device="cuda"), lens.to(torch.int32).cuda()
    qkv = torch.zeros((R, (heads + 2 * kv_heads) * dim), dtype=BF16, device="cuda")
    cos, sin = (a.cuda() for a in P.angles(256, dim))
    req = B.make_requests(table, starts, kv_len, tokens=R, max_new=1, max_len=256)
    split = lambda t: (t[:, :heads * dim].unflatten(1, (heads, dim)), *(c.unflatten(1, (kv_heads, dim)) for c in t[:, heads * dim:].chunk(2, 1)))  # noqa: E731

    def step(cache, q_out, out, ws):
        q, k, v = split(qkv)
        B.qail_kv_append(cache, req, k, v, q=q, q_out=q_out, cos=cos, sin=sin)
        B.qail_paged_attention(cache, req, q_out, out, dim ** -0.5, ws)

    def buffers(kv):
        cache = B.make_kv_cache(*kv)
        n = B.qail_paged_attention_workspace(cache, req, heads)
        return cache, torch.empty((R, heads, dim), dtype=BF16, device="cuda"), torch.empty((R, heads, dim), dtype=BF16, device="cuda"), \
            torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")

    mine, other = buffers(pools), buffers(twin)
    for b in (mine, other):    # both caches hold the token of before
        step(*b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*mine)
    side = torch.cuda.Stream()
    for i in range(6):
        qkv.normal_(generator=torch.Generator(device="cuda").manual_seed(30 + i))
        kv_len += 1
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            step(*other)
        torch.cuda.synchronize()
        assert torch.equal(mine[2], other[2]) and torch.equal(pools[0], twin[0]) and torch.equal(pools[1], twin[1])
        assert bool(mine[2].float().abs().sum() > 0)


# ----------------------------------------------------------------------------------------- adapters --

def adapter_case(shapes, M, n, r, seed, zero_weights=False):
    """Items and adapters on the device: random codes, or codes equal to their zero-points, so that the linear itself is zero."""
    items = []
    for i, (N, K, group) in enumerate(shapes):
        G = K // group
        q = torch.randint(-2 ** 31, 2 ** 31 - 1, (N, K // 8), generator=gen(seed + 10 * i), dtype=torch.int64).to(torch.int32)
        z = torch.randint(-2 ** 31, 2 ** 31 - 1, (N, -(-G // 8)), generator=gen(seed + 10 * i + 1), dtype=torch.int64).to(torch.int32)
        if zero_weights:
            q.fill_(0x77777777)
            z.fill_(0x77777777)
        s = (0.002 + 0.002 * torch.rand((N, G), generator=gen(seed + 10 * i + 2))).half()
        items.append(dict(N=N, K=K, group_size=group, qweight=q.cuda(), zeros=z.cuda(), scales=s.cuda(), x=P.normal((M, K), seed + 10 * i + 3).to(BF16).cuda(),
                          y=torch.full((M, N), math.nan, dtype=BF16, device="cuda"), A=P.normal((n, r, K), seed + 10 * i + 4, 0.05).to(BF16).cuda(),
                          B=P.normal((n, N, r), seed + 10 * i + 5, 0.05).to(BF16).cuda(), scaling=(0.5 + torch.rand((n,), generator=gen(seed + 10 * i + 6))).cuda()))
    return items


gen = P.gen


def run_adapters(B, items, rows, M):
    handle, ad = B.make_w4a16_items(items, M), B.make_adapters(items)
    ws = torch.full((B.qail_w4a16_adapters_workspace(handle, ad, len(items), M),), 255, dtype=torch.uint8, device="cuda")
    B.qail_w4a16_linear_adapters_batch(handle, ad, rows, len(items), M, ws)
    torch.cuda.synchronize()


def adapter_part(e, rows):
    """The adapters' part in 64 bits and the bound of its error before the last rounding: the down-projection's fp32 sums (K roundings), its
    two bf16 parts (2^-16), the up-projection's sums (2 r roundings) and the product with the scaling."""
    M, (n, r, K) = e["x"].shape[0], e["A"].shape
    part, tol = torch.zeros((M, e["N"]), dtype=P.F64), torch.zeros((M, e["N"]), dtype=P.F64)
    x = e["x"].double().cpu()
    for a in sorted(set(rows) & set(range(n))):
        at = torch.tensor([i for i, b in enumerate(rows) if b == a])
        A, Bf, c = e["A"][a].double().cpu(), e["B"][a].double().cpu(), e["scaling"][a].double().cpu()
        t, size = x[at] @ A.T, x[at].abs() @ A.abs().T
        part[at] = c * t @ Bf.T
        tol[at] = c * (K * 2 ** -24 * size + (2 ** -16 + 2 * r * 2 ** -24) * t.abs()) @ Bf.abs().T
    return part, tol


def some_rows(M, n, seed):
    """Runs of rows of one adapter, a few without any (-1, or a number that is none)."""
    g = gen(seed)
    rows = []
    while len(rows) < M:
        a = int(torch.randint(-1, n + 1, (1,), generator=g))
        rows += [a] * int(torch.randint(1, 1 + max(1, min(M, 40)), (1,), generator=g))
    return rows[:M]


ADAPTERS = [
    # (N, K, group) of each linear, rows, adapters, rank
    ([(64, 128, 64)], 1, 1, 8),
    ([(4096, 4096, 128)], 1, 5, 32),
    ([(520, 1024, 128), (33, 512, 64)], 3, 4, 16),          # a row of y that is not 16-byte aligned
    ([(256, 2048, 128)], 16, 16, 64),
    ([(1000, 1024, 128), (512, 2816, 128), (96, 512, 128)], 17, 3, 24),
    ([(768, 1024, 128)], 200, 6, 32),
    ([(129, 256, 128)], 300, 2, 40),
    ([(64, 72, 8)], 5, 3, 8),                               # K of no full step
    ([(64 + 8 * i, 256, 128) for i in range(11)], 4, 3, 16),   # more linears than share a launch
    ([(64, 72, 8), (256, 2816, 128), (520, 1024, 128)], 333, 5, 64),   # many rows: shares of K of different linears
    ([(96, 512, 128)], 260, 200, 16),                                  # ... of an adapter each
    ([(48, 9216, 128), (40, 256, 128)], 270, 3, 24),                   # ... the most shares and one
]


def linears(B, items, M):
    """What qail_w4a16_linear_batch gives."""
    handle = B.make_w4a16_items(items, M)
    need = B.qail_w4a16_batch_workspace(handle, len(items), M)
    B.qail_w4a16_linear_batch(handle, len(items), M, torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
    torch.cuda.synchronize()
    return [e["y"].clone() for e in items]


@pytest.mark.parametrize("zero_weights", [True, False])   # next to zero the adapters' part is nearly alone
@pytest.mark.parametrize("shapes,M,n,r", ADAPTERS)
def test_adapters_beside_the_linear(B, shapes, M, n, r, zero_weights):
    """Beside what qail_w4a16_linear_batch gives: its bits where a row has no adapter, its value and the adapters' part elsewhere."""
    items = adapter_case(shapes, M, n, r, 40 if zero_weights else 60, zero_weights)
    base = linears(B, items, M)
    for seed in (1, 2):
        rows = some_rows(M, n, seed) if seed == 1 else [(7 * i) % n for i in range(M)]    # ... and a row each
        run_adapters(B, items, torch.tensor(rows, dtype=torch.int32, device="cuda"), M)
        without = torch.tensor([not 0 <= a < n for a in rows])
        for e, y in zip(items, base):
            part, tol = adapter_part(e, rows)
            want = y.double().cpu() + part
            within(e["y"], want, 2 ** -8 * want.abs() + tol * (1 + 2 ** -7), (e["N"], seed))
            assert torch.equal(e["y"].cpu()[without], y.cpu()[without])
        first = [e["y"].clone() for e in items]
        run_adapters(B, items, torch.tensor(rows, dtype=torch.int32, device="cuda"), M)
        assert all(torch.equal(e["y"], y) for e, y in zip(items, first))


def test_adapters_do_not_reach_each_other(B):
    """An adapter of infinities and NaN beside others in the same tile of rows."""
    M, n, r = 12, 3, 16
    items = adapter_case([(200, 256, 128)], M, n, r, 80)
    rows = torch.tensor([0, 1, 2] * 4, dtype=torch.int32, device="cuda")
    run_adapters(B, items, rows, M)
    want = items[0]["y"].clone()
    items[0]["A"][1] = math.nan
    items[0]["B"][1, ::2] = math.inf
    run_adapters(B, items, rows, M)
    good = rows != 1
    assert torch.equal(items[0]["y"][good], want[good])
    assert not bool(torch.isfinite(items[0]["y"][~good].float()).all())


def test_adapters_in_a_graph(B):
    """Captured once, replayed with other rows: the adapters are chosen when the kernels run."""
    M, n, r = 6, 4, 16
    items = adapter_case([(256, 512, 128), (128, 256, 128)], M, n, r, 90)
    handle, ad = B.make_w4a16_items(items, M), B.make_adapters(items)
    ws = torch.empty(B.qail_w4a16_adapters_workspace(handle, ad, 2, M), dtype=torch.uint8, device="cuda")
    rows = torch.zeros(M, dtype=torch.int32, device="cuda")
    B.qail_w4a16_linear_adapters_batch(handle, ad, rows, 2, M, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.qail_w4a16_linear_adapters_batch(handle, ad, rows, 2, M, ws)
    for i in range(4):
        rows.copy_(torch.tensor([(i + j) % (n + 1) - 1 for j in range(M)], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = [e["y"].clone() for e in items]
        B.qail_w4a16_linear_adapters_batch(handle, ad, rows, 2, M, ws)
        torch.cuda.synchronize()
        assert all(torch.equal(e["y"], y) for e, y in zip(items, got))


# -------------------------------------------------------------------------------------- marshalling --

def test_native_marshalling_takes_plain_calls_with_the_same_results(B, monkeypatch):
    """Each of the five calls is taken by the compiled marshalling, on the current stream, and gives what the way through Python gives."""
    s = P.Step([2, 1], [30, 20], 4, 2, 64, 16, False, 61, pad=8)
    pools, keep = s.pools("cuda"), (s.table.cuda(), s.starts.cuda(), s.kv_len.cuda(), s.qkv.cuda())
    c, b = B.make_kv_cache(*pools), B.make_requests(*keep[:3], tokens=3, max_new=2, max_len=30)
    q, k, v = s.split(keep[3])
    cos, sin = (a.cuda() for a in P.angles(40, 64))
    x, w = P.normal((3, 256), 1).to(BF16).cuda(), P.normal((256,), 2).to(BF16).cuda()
    h, y, dx, q_out, out = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty((3, 4, 64), dtype=BF16, device="cuda"), \
        torch.empty((3, 4, 64), dtype=BF16, device="cuda")
    dw = torch.empty(256, device="cuda")
    codes, scale = torch.empty((3, 256), dtype=torch.int8, device="cuda"), torch.empty(3, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    items = adapter_case([(64, 128, 64)], 3, 2, 8, 70)
    handle, ad, rows = B.make_w4a16_items(items, 3), B.make_adapters(items), torch.tensor([0, 1, -1], dtype=torch.int32, device="cuda")
    errors = torch.zeros(1, dtype=torch.int32, device="cuda")
    outputs = [h, y, dx, q_out, out, dw, codes, scale, pools[0], pools[1], items[0]["y"]]

    def native():
        return [B._rmsnorm_native(x, w, 1e-5, x, h, y, codes, scale), B._rmsnorm_backward_native(x, w, 1e-5, h, dx, dw, ws, y),
                B._kv_append_native(c, b, k, v, q, q_out, cos, sin, errors), B._paged_attention_native(c, b, q_out, out, 0.125, None, errors),
                B._paged_attention_native(c, B.make_requests(keep[0][:1], keep[1][:2], keep[2][:1], tokens=1, max_new=1, max_len=30), q[:1], out[:1], 0.125, ws, None),
                B._paged_attention_native(c, b, q_out, out, 0.125, ws, None), B._adapters_batch_native(handle, ad, rows, 1, 3, ws)]

    def python():
        B.qail_rmsnorm(x, w, 1e-5, residual=x, residual_out=h, y=y, y_s8=codes, y_scale=scale)
        B.qail_rmsnorm_backward(x, w, 1e-5, h, dx, dw, ws, dres=y)
        B.qail_kv_append(c, b, k, v, q=q, q_out=q_out, cos=cos, sin=sin, errors=errors)
        B.qail_paged_attention(c, b, q_out, out, 0.125, None, errors)
        B.qail_w4a16_linear_adapters_batch(handle, ad, rows, 1, 3, ws)

    assert native() == [B.QAIL_OK] * 7
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]
    for name in ("_rmsnorm_native", "_rmsnorm_backward_native", "_kv_append_native", "_paged_attention_native", "_adapters_batch_native"):
        monkeypatch.setattr(B, name, B._not_plain)
    for t in outputs[:8] + outputs[10:]:
        t.zero_()
    python()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs[:8] + outputs[10:], want[:8] + want[10:]))
    assert torch.equal(pools[0].view(torch.int16), want[8].view(torch.int16)) and errors.item() == 0
    monkeypatch.undo()
    # on the stream that is current
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for t in outputs[:2]:
            t.zero_()
        assert B._rmsnorm_native(x, w, 1e-5, x, h, y, codes, scale) == B.QAIL_OK
    side.synchronize()
    assert torch.equal(h, want[0]) and torch.equal(y, want[1])
    # errors come back as the library's
    with pytest.raises(B.QailError):
        B.qail_rmsnorm(x, w, -1.0, y=y)
    assert B._rmsnorm_native(x.float(), w, 1e-5, None, None, y, None, None) is None
    with pytest.raises(ValueError, match="bfloat16"):
        B.qail_rmsnorm(x.float(), w, 1e-5, y=y)
    with pytest.raises(ValueError, match="heads of a token must be contiguous"):
        B.qail_paged_attention(c, b, q.transpose(1, 2).contiguous().transpose(1, 2), out, 0.125)
