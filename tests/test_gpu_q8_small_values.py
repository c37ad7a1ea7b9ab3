"""One new token over 8-bit pages whose values lie next to the smallest that a page holds.

A weight p times a value's power of two 2^e becomes a bf16 (bf16 queries; off by 2^-134 at most
below the normal numbers) or three (fp32 queries; the third cut off to whole 2^-133): with codes of
at most 127 < 2^7, n keys and l the sum of the weights over the largest, an output is off by another
2^-126 n / l.  Rows of prompts take the values as they are and have the ordinary tolerances."""
import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import PoolCase, attention64, cu
from tests.q8_cases import Q8Pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("prompts", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("by", [2.0 ** -100, 2.0 ** -110, 2.0 ** -114, 2.0 ** -117])
def test_small_values(by, hd, prompts, dtype):
    n = 300
    case = PoolCase([n], 2, hd, 16)
    case.values[0] = (case.values[0].float() * by).to(torch.bfloat16)
    for j in range(-(-n // 16)):
        m = min(16, n - j * 16)
        case.v[int(case.table[0, j]), :, :m] = case.values[0][j * 16: j * 16 + m].transpose(0, 1)
    pool = Q8Pool(case)
    g = torch.Generator().manual_seed(4)
    q = torch.randn((1, 4, hd), generator=g).to(dtype)
    k, v, ke, ve, lens, table = pool.device()
    out, lse = torch.empty_like(q).cuda(), torch.empty((1, 4), device="cuda")
    kw = dict(cu_q=cu([1]).cuda()) if prompts else {}
    B.aio_q8_attention(q.cuda(), k, v, ke, ve, lens, table, out, lse=lse, **kw)
    want, l64, tol, ltol = attention64(q, case.keys, case.values, [1], [n])
    assert ((lse.double().cpu() - l64).abs() <= ltol).all()
    s = (q[0].double()[None] * case.keys[0].double().repeat_interleave(2, dim=1)).sum(-1) * hd ** -0.5
    weights = torch.exp(l64[0] - s.amax(0))
    more = 0 if prompts else 2.0 ** -126 * n / weights[:, None]
    err = (out.double().cpu() - want).abs()[0]
    assert (err <= tol[0] + more + 2.0 ** -134).all(), float((err / (tol[0] + more)).max())
