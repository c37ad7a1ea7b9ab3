"""Values that are not finite under weights that underflow: whether the keys are split
over workgroups or not, the outputs that see such a value are not finite, and no others."""
import math

import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import attention64, check_attention, cu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n", [200, 3000, 20000])
@pytest.mark.parametrize("rows", [None, 1, 5])  # None: one new token
@pytest.mark.parametrize("far", [-300.0, -30.0])  # a weight of e^-300 is 0 in fp32
def test_far_below_the_maximum(far, rows, n, hd, dtype):
    g = torch.Generator().manual_seed(n)
    nq = rows or 1
    half = n // 2 // 64 * 64
    k = torch.zeros((n, 1, hd), dtype=torch.bfloat16)
    k[:half, 0, 0] = far
    v = torch.randn((n, 1, hd), generator=g).to(torch.bfloat16)
    q = torch.zeros((nq, 2, hd), dtype=dtype)
    q[:, :, 0] = 1
    want = [t.clone() for t in attention64(q, [k], [v], [nq], [n], scale=1.0)]
    odd = {5: math.inf, 9: math.nan, 20: -math.inf}
    for i, (d, x) in enumerate(odd.items()):
        v[(10, 70, half - 1)[i], 0, d] = x
    page = 16
    pages = -(-n // page)
    kp, vp = (torch.cat((t, torch.zeros((pages * page - n, 1, hd), dtype=t.dtype)))
              .reshape(pages, page, 1, hd).transpose(1, 2).contiguous().cuda() for t in (k, v))
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    got = []
    kw = dict(scale=1.0)
    if rows:
        kw["cu_q"] = cu([nq]).cuda()
        out, lse = torch.empty_like(q).cuda(), torch.empty((nq, 2), device="cuda")
        B.aio_packed_attention(q.cuda(), k.cuda(), v.cuda(), cu([nq]).cuda(), cu([n]).cuda(), out,
                               lse=lse, scale=1.0)
        got.append((out, lse))
    for max_len in (n, 1 << 20):  # (a bound that is far too large splits differently)
        need = B.aio_attn_workspace_bytes(1, nq, max_len, 2, 1, hd, prompts=rows is not None)
        assert (need > 0) == (rows is not None or max_len > 512)
        out, lse = torch.empty_like(q).cuda(), torch.empty((nq, 2), device="cuda")
        B.aio_paged_attention(q.cuda(), kp, vp, lens, table, out, lse=lse, max_len=max_len, **kw)
        got.append((out, lse))
    for out, lse in got:
        out = out.cpu()
        for d in odd:
            assert not torch.isfinite(out[:, :, d]).any(), (d, out[:, :, d])
            out[:, :, d] = want[0][:, :, d].to(dtype)
        check_attention(out, lse.cpu(), want)
