"""GPU tests of how many bits the serving operators keep between their inputs and the rounding of their outputs."""
import math

import pytest
import torch

from tests import serve_reference as P
from tests.helpers import ensure_built
from tests.test_gpu_serve import attention, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    return ensure_built()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page", [([1], [200], 4, 4, 128, 32), ([1], [3000], 4, 2, 64, 32), ([1] * 3, [2500, 40, 900], 16, 1, 128, 128),
                                                              ([5, 2, 16], [5, 90, 300], 2, 2, 128, 16), ([40, 2], [40, 300], 2, 1, 64, 64)])
def test_few_rows_keep_more_of_p_than_bf16(B, new, lens, heads, kv_heads, dim, page, eight):
    """Of requests with up to 16 rows a head of the cache: p is in two bf16 parts, of which 2^-16 may be lost; else as serve_reference.attend counts."""
    s = P.Step(new, lens, heads, kv_heads, dim, page, eight, 3000 + page, pad=8)
    scale = 1 / math.sqrt(dim)
    want, tol = P.attend(s, scale)
    few = torch.zeros(s.tokens, dtype=torch.bool)
    for r, n in enumerate(new):
        if n * heads // kv_heads <= 16:
            few[int(s.starts[r]):int(s.starts[r + 1])] = True
    spread = torch.zeros_like(want)     # sum of p |v|
    real = s.real
    s.real = lambda r, i: real(r, i).abs() if i else real(r, i)
    spread = P.attend(s, scale)[0]
    s.real = real
    tol = tol - (2 ** -8 - 2 ** -16) * spread
    within(attention(B, s, scale)[few.cuda()], want[few], tol[few])
