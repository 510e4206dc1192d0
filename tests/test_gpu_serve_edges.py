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


# q_start that descends behind the last row, lengths of requests that wait; with few rows, with many, with keys that are divided among blocks
BAD = [([5, 0, 0], [20, 10, 30], 40), ([5, 0, 0], [20, 10, 30], 3000), ([70, 0, 0], [100, 10, 30], 100), ([70, 0, 3], [100, 10, 2000], 2000)]


@pytest.mark.parametrize("new,lens,max_len", BAD)
@pytest.mark.parametrize("what,index,value", [("starts", 2, -1), ("starts", 3, 1), ("lens", 1, 10 ** 6), ("lens", 1, -1), ("lens", 1, 2 ** 31 - 1), ("lens", 1, -2 ** 31)])
def test_what_is_bad_where_no_row_looks_is_counted(B, new, lens, max_len, what, index, value):
    for append in (False, True):
        s = P.Step(new, lens, 2, 1, 64, 16, False, 23)
        table = torch.nn.functional.pad(s.table, (0, 200), value=-7).cuda()    # room for max_len
        starts, kv_len = s.starts.cuda(), s.kv_len.cuda()
        (starts if what == "starts" else kv_len)[index] = value
        k, v, _, _ = s.pools("cuda")
        cache, req = B.make_kv_cache(k, v), B.make_requests(table, starts, kv_len, tokens=s.tokens, max_new=max(new), max_len=max_len)
        errors, out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((s.tokens, 2, 64), dtype=BF16, device="cuda")
        q, nk, nv = s.split(s.qkv.cuda())
        if append:
            B.qail_kv_append(cache, req, nk, nv, errors=errors)
        else:
            n = B.qail_paged_attention_workspace(cache, req, 2)
            B.qail_paged_attention(cache, req, q, out, 0.125, torch.empty(max(n, 256), dtype=torch.uint8, device="cuda"), errors=errors)
        torch.cuda.synchronize()
        assert errors.item() > 0, append
