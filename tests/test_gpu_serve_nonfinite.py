"""GPU tests of infinities and NaN in what the serving operators see: they come out where the formulas say so, whatever the launches are, and
nowhere else.  Tolerances are those of tests/test_gpu_serve.py."""
import math

import pytest
import torch

from tests import serve_reference as P
from tests.helpers import ensure_built
from tests.test_gpu_serve import adapter_case, adapter_part, attention, linears, run_adapters, within

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    return ensure_built()


# few rows and many, each with keys that one block takes and with keys that are divided among blocks, beside a request of the other kind,
# grouped heads, heads of either size; keys `first` to `last` - 1 are whole shares of blocks where they are divided (256 keys, or 448 of many rows)
SEEN = [
    # new, lens, heads, kv_heads, dim, page, first, last
    ([1], [200], 4, 2, 128, 32, 64, 100),
    ([1], [3000], 4, 2, 128, 32, 256, 1280),
    ([1] * 3, [2500, 40, 900], 16, 1, 128, 128, 512, 1536),
    ([1, 3], [4000, 3000], 8, 8, 64, 64, 1024, 3072),
    ([40, 2], [40, 30], 2, 1, 64, 32, 0, 1),
    ([100, 3], [2100, 1500], 8, 8, 64, 256, 448, 1344),
    ([40], [2600], 8, 2, 128, 64, 448, 1792),
]


def nan_rows(B, s, poison, rows):
    """`rows` ([tokens, heads] of truth values) come out as NaN, the others as they are without the poison."""
    scale = 1 / math.sqrt(s.dim)
    want, tol = P.attend(s, scale)
    poison()
    out = attention(B, s, scale).cpu()
    assert bool(torch.isnan(out[rows]).all())
    within(out[~rows], want[~rows], tol[~rows])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page,first,last", SEEN)
def test_nan_of_a_query(B, new, lens, heads, kv_heads, dim, page, first, last, eight):
    """One value of one head of the first request's last token."""
    s = P.Step(new, lens, heads, kv_heads, dim, page, eight, 2000 + first, pad=8)
    rows = torch.zeros((s.tokens, heads), dtype=torch.bool)
    rows[new[0] - 1, heads - 1] = True
    nan_rows(B, s, lambda: s.split(s.qkv)[0][new[0] - 1, heads - 1].__setitem__(5, math.nan), rows)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page,first,last", SEEN)
def test_nan_of_all_keys_of_a_share(B, new, lens, heads, kv_heads, dim, page, first, last, eight):
    """Of one head of the cache, in keys that all rows of the first request see."""
    s = P.Step(new, lens, heads, kv_heads, dim, page, eight, 2100 + first, pad=8)
    rows = torch.zeros((s.tokens, heads), dtype=torch.bool)
    rows[:new[0], :heads // kv_heads] = True

    def poison():
        k = s.values[0][0]
        (k[1] if eight else k)[0, first:last] = math.nan

    nan_rows(B, s, poison, rows)


# ---------------------------------------------------------------------------- values that are infinite --

# lengths that end inside a tile of keys and at its end, few rows and many, undivided and divided
LAST = [([1], [90], 4, 2, 128, 32), ([1], [96], 4, 2, 128, 32), ([5], [91], 2, 1, 64, 16), ([1, 1], [3001, 2999], 8, 8, 64, 64), ([70], [70], 2, 1, 128, 16),
        ([64], [128], 2, 1, 128, 16), ([40], [2601], 8, 2, 128, 64), ([100, 3], [2100, 1501], 8, 8, 64, 256)]


@pytest.mark.parametrize("value", [math.inf, -math.inf])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page", LAST)
def test_an_infinite_value_is_infinite_for_those_who_see_it(B, new, lens, heads, kv_heads, dim, page, eight, value):
    """In each request's last token's value: the rows of that token alone see it, however many slots of a tile lie behind it."""
    s = P.Step(new, lens, heads, kv_heads, dim, page, eight, 2300 + lens[0], pad=8)
    scale = 1 / math.sqrt(dim)
    for r in range(len(new)):
        v = s.values[r][1]
        if eight:
            v[0][:, -1] = torch.where(v[0][:, -1] == 0, 1, v[0][:, -1])    # zero times an infinity is NaN
    want, tol = P.attend(s, scale)
    sees = torch.zeros((s.tokens, heads, dim), dtype=torch.bool)
    for r in range(len(new)):
        row = int(s.starts[r + 1]) - 1
        if eight:
            v = s.values[r][1]
            v[1][:, -1] = abs(value)
            want[row] = (v[0][:, -1].double() * math.inf).repeat_interleave(heads // kv_heads, 0)
            sees[row] = True
        else:
            s.values[r][1][:, -1, 7] = value
            want[row, :, 7] = value
            sees[row, :, 7] = True
    out = attention(B, s, scale).double().cpu()
    assert torch.equal(out[sees], want[sees])
    if not sees.all():
        within(out[~sees], want[~sees], tol[~sees])


@pytest.mark.parametrize("first", [0, 0.3, 0.6])
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page", LAST)
def test_an_infinite_value_of_a_key_in_front(B, new, lens, heads, kv_heads, dim, page, first):
    """One value of one key of each request, at the beginning or further on: infinite in the rows that see it, which are right beside it."""
    s = P.Step(new, lens, heads, kv_heads, dim, page, False, 2500 + lens[0], pad=8)
    scale = 1 / math.sqrt(dim)
    want, tol = P.attend(s, scale)
    sees = torch.zeros((s.tokens, heads, dim), dtype=torch.bool)
    for r, (n, length) in enumerate(zip(new, lens)):
        key = int(first * length)
        s.values[r][1][:, key, 5] = math.inf
        sees[int(s.starts[r]) + max(0, key - (length - n)):int(s.starts[r + 1]), :, 5] = True
    out = attention(B, s, scale).double().cpu()
    assert bool((out[sees] == math.inf).all())
    within(out[~sees], want[~sees], tol[~sees])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page", LAST + [([1], [1], 1, 1, 64, 16), ([200], [150], 4, 4, 128, 64)])
def test_scores_of_minus_infinity_alone_are_nan(B, new, lens, heads, kv_heads, dim, page, eight):
    """A row whose keys all have a score of minus infinity has no largest one, unlike a row without keys, which is zeros."""
    s = P.Step(new, lens, heads, kv_heads, dim, page, eight, 2400 + lens[0], pad=8)
    scale = 1 / math.sqrt(dim)
    want, tol = P.attend(s, scale)
    q, _, _ = s.split(s.qkv)
    q[:, 0] = q[:, 0].abs() + 1    # the first head's scores of keys below zero are below zero
    k = s.values[0][0]
    if eight:
        k[0][0] = -1
        k[1][0] = math.inf
    else:
        k[0] = -math.inf
    rows = torch.zeros((s.tokens, heads), dtype=torch.bool)
    rows[max(0, new[0] - lens[0]):new[0], 0] = True
    others = torch.ones_like(rows)
    others[:, 0] = False                                   # its queries are others
    others[:new[0], :heads // kv_heads] = False            # these read the same keys
    out = attention(B, s, scale).cpu()
    assert bool(torch.isnan(out[rows]).all())
    if others.any():
        within(out[others], want[others], tol[others])
    assert not out[:max(0, new[0] - lens[0]), 0].any()


# -------------------------------------------------------------------------------- a cache of bytes --

@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_head_that_is_not_finite_has_a_step_of_nan(B, dim, value):
    """One value of a key, one of a value, a whole head: their tokens are NaN when they are read; every other code and step is what it is without them."""
    s = P.Step([3, 2], [20, 40], 2, 2, dim, 16, True, 11)
    cos, sin = (t.cuda() for t in P.angles(40, dim))
    clean, qkv = s.qkv.cuda(), s.qkv.cuda()
    _, k, v = s.split(qkv)
    k[0, 1, dim - 1] = value
    v[4, 0, 2] = value
    k[2, 0] = value
    v[2, 1] = value
    got = []
    for t in (clean, qkv):
        pools = s.pools("cuda")
        keep = s.table.cuda(), s.starts.cuda(), s.kv_len.cuda()
        q, nk, nv = s.split(t)
        out = torch.empty((s.tokens, 2, dim), dtype=BF16, device="cuda")
        errors = torch.zeros(1, dtype=torch.int32, device="cuda")
        req = B.make_requests(*keep, tokens=s.tokens, max_new=3, max_len=40)
        B.qail_kv_append(B.make_kv_cache(*pools), req, nk, nv, q=q, q_out=out, cos=cos, sin=sin, errors=errors)
        torch.cuda.synchronize()
        assert errors.item() == 0
        got.append([p.cpu() for p in pools])
    bad = torch.zeros((2,) + got[0][2].shape, dtype=torch.bool)    # of keys and of values: [page, head, slot]
    at = [(int(s.table[r, p // 16]), p % 16) for r, p in P.positions(s)]
    for which, token, head in ((0, 0, 1), (1, 4, 0), (0, 2, 0), (1, 2, 1)):
        bad[which, at[token][0], head, at[token][1]] = True
    for which in range(2):
        codes, step = got[1][which], got[1][2 + which]
        assert bool(torch.isnan(step[bad[which]]).all())
        assert torch.equal(codes[~bad[which]], got[0][which][~bad[which]])
        assert torch.equal(step[~bad[which]].view(torch.int32), got[0][2 + which][~bad[which]].view(torch.int32))


# ------------------------------------------------------------------------------------ codes of a norm --

@pytest.mark.parametrize("where", ["x", "residual", "weight"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("K", [64, 1000, 2048, 4096, 16384])
def test_codes_of_a_norm_of_what_is_not_finite(B, K, value, where):
    """The scale of a row with an infinity or NaN is NaN (the weight's is in every row); other rows keep their bits."""
    M = 5
    x, res, w = P.normal((M, K), 1).to(BF16).cuda(), P.normal((M, K), 2).to(BF16).cuda(), (1 + P.normal((K,), 3, 0.2)).to(BF16).cuda()
    got = []
    for poisoned in (False, True):
        if poisoned:
            if where == "weight":
                w[K - 3] = value
            else:
                (x if where == "x" else res)[3, K - 3] = value
        codes, scale = torch.empty((M, K), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
        B.qail_rmsnorm(x, w, 1e-5, residual=res, y_s8=codes, y_scale=scale)
        got.append((codes.cpu(), scale.cpu()))
    rows = torch.full((M,), where == "weight")
    rows[3] = True
    assert bool(torch.isnan(got[1][1][rows]).all())
    assert torch.equal(got[1][0][~rows], got[0][0][~rows]) and torch.equal(got[1][1][~rows], got[0][1][~rows])


# ----------------------------------------------------------------------------------------- adapters --

@pytest.mark.parametrize("shapes,M,n,r", [([(256, 512, 128)], 3, 3, 8), ([(520, 1024, 128), (33, 512, 64)], 20, 2, 16), ([(96, 512, 128)], 100, 4, 64),
                                          ([(129, 256, 128), (64, 2048, 128)], 350, 3, 40)])
def test_infinities_of_an_adapter_are_what_the_products_say(B, shapes, M, n, r):
    """A down-projection beyond fp32, and infinities among B's values: y is infinite with the sign of their product; what they do not reach stays."""
    items = adapter_case(shapes, M, n, r, 120, zero_weights=True)
    rows = [i % (n + 1) - 1 for i in range(M)]
    device_rows = torch.tensor(rows, dtype=torch.int32, device="cuda")
    row = rows.index(1)
    for kind in ("t", "B"):
        for e in items:
            if kind == "t":    # t[row][2] = 1e25 * 1e25 and what is finite beside it; every other t is finite
                e["A"][:, :, 7] = 0
                e["A"][1, 2, 7] = 1e25
                e["x"][:, 7] = 0
                e["x"][row, 7] = 1e25
            else:
                e["A"][1, 2, 7] = 0
                e["x"][row, 7] = 0
                e["B"][1, 1::3, 4] = math.inf
                e["B"][1, 2::3, 4] = -math.inf
        base = linears(B, items, M)
        run_adapters(B, items, device_rows, M)
        for e, linear in zip(items, base):
            y = e["y"].double().cpu()
            part, tol = adapter_part(dict(e, B=torch.where(torch.isfinite(e["B"]), e["B"], 0), x=torch.where(e["x"].float().abs() < 1e20, e["x"], 0)), rows)
            want = linear.double().cpu() + part
            if kind == "t":
                want[row] = e["B"][1, :, 2].double().cpu() * math.inf
            else:
                t = e["x"].double().cpu() @ e["A"][1, 4].double().cpu()
                for m in [i for i, a in enumerate(rows) if a == 1]:
                    want[m, 1::3] = t[m] * math.inf
                    want[m, 2::3] = -t[m] * math.inf
            inf = torch.isinf(want)
            assert not torch.isnan(want).any() and torch.equal(y[inf], want[inf]), kind
            assert bool(((y - want).abs() <= 2 ** -8 * want.abs() + tol * (1 + 2 ** -7))[~inf].all()), kind
