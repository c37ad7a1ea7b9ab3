"""Thousands of groups in one call: more than two levels of the 64-wide search for a tile's and a
sequence's group."""
import pytest
import torch

from tests.paged_cases import attention64, check_attention
from tests.test_gpu_prefix_attention import BF16, F32, Grouped, rows

pytestmark = pytest.mark.gpu


CASES = [(w, t, m, False) for w in (1, 2, 5) for t in (F32, BF16) for m in (False, True)]


# (quantising on the CPU is what takes time)
@pytest.mark.parametrize("width,dtype,prompts,q8", CASES + [(2, F32, False, True),
                                                            (2, BF16, True, True)])
def test_thousands_of_groups(width, dtype, prompts, q8):
    n = 4500 * width if width < 3 else 9000
    k_len = [64 + (7 * i) % 30 if i % 11 else 5 for i in range(n)]
    groups = [(i, min(i + width, n), 64) for i in range(0, n, width) if i % 13]
    p = Grouped(k_len, groups, 1, 64, page=32, q8=q8)
    ql = [(1 + i % 3 if i % 17 else 0) for i in range(n)] if prompts else [1] * n
    q = rows(sum(ql), 2, 64, dtype)
    first = [0]
    for v in ql:
        first.append(first[-1] + v)
    at = sorted(set(list(range(0, n, 97)) + list(range(40)) + list(range(n - 40, n))))
    at = [i for i in at if ql[i]]
    pick = torch.cat([torch.arange(first[i], first[i + 1]) for i in at])
    c = p.case
    want = attention64(q[pick], [c.keys[i] for i in at], [c.values[i] for i in at],
                       [ql[i] for i in at], [k_len[i] for i in at])
    for kw in (dict(max_len=93, max_prefix=64), dict()):
        out, l = p.run(q, ql if prompts else None, **kw)
        check_attention(out[pick.cuda()], l[pick.cuda()], want, str(kw))
        assert torch.isfinite(out).all()
