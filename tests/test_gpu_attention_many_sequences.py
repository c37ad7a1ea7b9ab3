"""Prompt rows of more sequences than a wave looks at together, most of them without rows:
every row is computed, by its own sequence's keys."""
import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import attention64, check_attention

pytestmark = pytest.mark.gpu


def lengths(kind, n, g):
    if kind == "ones":
        return torch.ones(n, dtype=torch.int64)
    if kind == "few":  # nearly all are empty, the rest up to 600 rows
        q = torch.zeros(n, dtype=torch.int64)
        at = torch.randperm(n, generator=g)[:9]
        q[at] = torch.tensor([1, 2, 127, 128, 129, 255, 256, 257, 600])
        return q
    q = torch.randint(0, 4, (n,), generator=g)
    q[:: 97] = 200
    return q


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind,n,H,Hkv,wide", [
    ("ones", 65, 2, 1, False), ("ones", 4097, 4, 4, False), ("few", 70, 4, 2, False),
    ("few", 5000, 4, 2, False), ("few", 1 << 20, 4, 2, False), ("mixed", 64 * 64 + 1, 3, 1, False),
    ("mixed", 3000, 64, 8, True)])
def test_every_row(kind, n, H, Hkv, wide, dtype):
    g = torch.Generator().manual_seed(n)
    ql = lengths(kind, n, g)
    cu = torch.cat((torch.zeros(1, dtype=torch.int64), ql.cumsum(0)))
    rows, hd = int(cu[-1]), 64
    k = torch.randn((rows, Hkv, hd), generator=g).to(torch.bfloat16)
    v = torch.randn((rows, Hkv, hd), generator=g).to(torch.bfloat16)
    q = torch.randn((rows + 1, H, hd), generator=g).to(dtype)
    assert wide == (rows * H // Hkv // 256 * Hkv >= 1024)
    c = cu.int().cuda()
    out = torch.full_like(q, 9.0).cuda()
    B.aio_packed_attention(q.cuda(), k.cuda(), v.cuda(), c, c, out)
    out = out.cpu()
    assert (out[:rows] != 9).any(-1).all() and (out[rows:] == 9).all()
    # rows that are first in their sequence see one key, their own: its weight, the sum, its
    # inverse, the product and the output round
    seqs = torch.nonzero(ql)[:, 0]
    first = cu[seqs]
    one = v[first].repeat_interleave(H // Hkv, 1).float()
    off = 2.0 ** -7 + 2.0 ** -16 if dtype == torch.bfloat16 else 2.0 ** -22
    assert ((out[first].float() - one).abs() <= off * one.abs()).all()
    # the last rows of the longest and of the last sequences
    some = torch.cat((seqs[ql[seqs].argsort()[-4:]], seqs[-3:])).tolist()
    for i in some:
        a, b = int(cu[i]), int(cu[i + 1])
        ref = attention64(q[b - 1: b], [k[a:b]], [v[a:b]], [1], [b - a])
        check_attention(out[b - 1: b], None, ref, (kind, i))
