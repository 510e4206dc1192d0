"""GPU tests of infinities and NaN in what the serving operators see: they come out where the formulas say so, whatever the launches are, and
nowhere else.  Tolerances are those of tests/test_gpu_serve.py."""
import math

import pytest
import torch

from tests import serve_reference as P
from tests.helpers import ensure_built
from tests.test_gpu_serve import attention, within

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
