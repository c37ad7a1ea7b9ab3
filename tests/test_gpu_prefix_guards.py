"""Attention of groups writes its outputs, its log-sum-exps and its workspace and nothing beside
them, whatever the groups' boundaries and lengths hold; codes that an append writes, read back."""
import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import PoolCase, check_attention, cu
from tests.q8_cases import Q8Pool
from tests.test_gpu_prefix_attention import BF16, F32, Grouped, i32, rows

pytestmark = pytest.mark.gpu

GUARD = 1 << 16  # bytes before and behind each buffer


class Guarded:
    """A buffer of exactly so many bytes between two of a pattern."""

    def __init__(self, n):
        self.n = n
        i = torch.arange(n + 2 * GUARD, dtype=torch.int64, device="cuda")
        self.pattern = ((i * 2654435761) >> 7 & 255).to(torch.uint8)
        self.all = self.pattern.clone()

    def view(self, dtype, *shape):
        return self.all[GUARD: GUARD + self.n].view(dtype).view(shape)

    def untouched(self):
        return (torch.equal(self.all[:GUARD], self.pattern[:GUARD]) and
                torch.equal(self.all[GUARD + self.n:], self.pattern[GUARD + self.n:]))


BIG = (1 << 31) - 1
SENSELESS = [
    ([0, 1 << 30], [280]), ([-5, 4], [1 << 30]), ([3, 0], [280]), ([4, 4], [100]), ([0, 4], [-1]),
    ([0, 4], [BIG]), ([0, 3, 1, 4], [280, 64, 200]), ([2, 2, 2, 2], [64, 64, 64]),
    ([-1 << 31, BIG], [BIG]), ([4, 3, 2, 1, 0], [64, 128, 192, 256]), ([1, BIG, 0, 2], [BIG, 64, 300]),
    ([0, 1, 1, 40, 3], [64, 280, BIG, 128])]


# steps, steps of many columns, prompt rows, prompt rows in tiles of 256 (over 8-bit pages)
@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("dtype,ql,H,hd,n", [
    (F32, None, 4, 64, 4), (BF16, None, 32, 128, 14), (F32, [4, 9, 1, 30], 4, 64, 4),
    (BF16, [4, 9, 1, 30], 4, 128, 4), (BF16, [290, 100, 290, 340], 16, 64, 4)])
def test_nothing_beside_the_buffers_is_written(dtype, ql, H, hd, n, q8):
    k_len = [300 + 10 * (i % 4) for i in range(n)]
    p = Grouped(k_len, [(0, n, 280)], 2, hd, q8=q8)
    q = rows(sum(ql) if ql else n, H, hd, dtype)
    want = p.ref(q, ql)
    right = p.cu_seqs, p.prefix
    kv, qd = [t.clone() for t in p.kv], q.cuda()
    kw = dict(max_len=max(k_len), max_prefix=280)
    if ql:
        kw["cu_q"] = cu(ql).cuda()
    ids = [t.clone() for t in (p.lens, p.table)]

    def one(groups, prefix):
        p.cu_seqs, p.prefix = groups, prefix
        out = Guarded(q.numel() * q.element_size())
        lse = Guarded(q.shape[0] * H * 4)
        need = B.aio_prefix_workspace_bytes(n, q.shape[0], kw["max_len"], len(prefix), 280, H, 2, hd,
                                            prompts=ql is not None)
        ws = Guarded(need)
        o, l = out.view(dtype, *q.shape), lse.view(F32, q.shape[0], H)
        p.call(qd, o, lse=l, ws=ws.view(torch.uint8, need), **kw)
        torch.cuda.synchronize()
        for what, g in (("out", out), ("lse", lse), ("ws", ws)):
            assert g.untouched(), (what, groups.tolist(), prefix.tolist())
        assert torch.equal(qd.cpu(), q)
        for a, b in zip([*p.kv, p.lens, p.table], kv + ids):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        return o, l

    check_attention(*one(*right), want)
    for c, m in SENSELESS:
        one(i32(c), i32(m))
    check_attention(*one(*right), want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [64, 128])
def test_appended_codes_read_back(hd, dtype):
    """Each element within A / 127 of its row's largest magnitude A, or 2^-120 where that is more."""
    n = 60
    g = torch.Generator().manual_seed(3)
    x = torch.randn((2, n, 3, hd), generator=g) * torch.exp2(
        torch.randint(-125, 120, (2, n, 3, 1), generator=g).float())
    x = x.to(dtype)
    pool = Q8Pool(PoolCase([n], 3, hd, 16))
    k, v, ke, ve, lens, table = pool.device()
    B.aio_q8_append(x[0].cuda(), x[1].cuda(), k, v, ke, ve, lens, table, cu_q=cu([n]).cuda())
    at = pool.case.table[0].tolist()
    for w, (codes, exps) in enumerate(((k, ke), (v, ve))):
        codes, exps = codes.cpu(), exps.cpu()
        for i in range(n):
            c, e = codes[at[i // 16], :, i % 16], exps[at[i // 16], :, i % 16]
            assert ((e >= 8) & (e <= 248)).all() and (c >= -127).all()
            back = torch.ldexp(c.double(), e.double()[:, None] - 127)
            row = x[w, i].double()
            most = (row.abs().amax(-1, keepdim=True) / 127).clamp_min(2.0 ** -120)
            assert ((back - row).abs() <= most).all()
