"""GPU tests of steps at the borders of what the serving operators take: many requests that wait, arrays that are bad where no row looks."""
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


def test_many_requests_wait(B):
    """Two requests with rows among 20000: the launches are those of the rows."""
    new, lens = [0] * 20000, [0] * 20000
    for r, n, length in ((3, 40, 700), (19998, 5, 90)):
        new[r], lens[r] = n, length
    s = P.Step(new, lens, 4, 2, 64, 64, False, 31)
    want, tol = P.attend(s, 1 / math.sqrt(64))
    within(attention(B, s, 1 / math.sqrt(64)), want, tol)
