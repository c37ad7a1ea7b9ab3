"""Rows appended to pages and pages copied, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import PoolCase, cu

pytestmark = pytest.mark.gpu


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


def expect_append(case, kr, vr, ql, lens, max_len=1 << 30):
    """The pool after the append, on the CPU."""
    pool = case.pool.clone()
    if case.layout == "plain":
        k, v = pool[0], pool[1]
    else:
        k, v = pool[:, 0, :, : case.page], pool[:, 1, :, : case.page]
    r = 0
    for i, (q, n) in enumerate(zip(ql, lens)):
        for j in range(q):
            pos = n - q + j
            if 0 <= pos < min(max_len, case.table.shape[1] * case.page):
                pg = int(case.table[i, pos // case.page])
                if 0 <= pg < case.n_pages:
                    k[pg, :, pos % case.page] = kr[r + j].to(torch.bfloat16)
                    v[pg, :, pos % case.page] = vr[r + j].to(torch.bfloat16)
        r += q
    return pool


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("Hkv,hd,page,layout", [
    (8, 128, 16, "plain"), (1, 64, 8, "plain"), (3, 64, 64, "interleaved"),
    (32, 128, 256, "interleaved")])
def test_append(Hkv, hd, page, layout, dtype):
    ql, kl = [1, 0, 7, 20, 3], [1, 30, 40, 20, 257]
    case = PoolCase(kl, Hkv, hd, page, holes=[(2, 1)], layout=layout)
    g = torch.Generator().manual_seed(3)
    n = sum(ql) + 2  # two rows of no sequence
    kr = torch.randn((n, Hkv, hd), generator=g).to(dtype)
    vr = torch.randn((n, Hkv, hd), generator=g).to(dtype)
    k, v, lens, table = case.device()
    whole = k._base if k._base is not None else k
    B.aio_page_append(kr.cuda(), vr.cuda(), k, v, lens, table, cu_q=cu(ql).cuda())
    torch.cuda.synchronize()
    assert same_bits(whole.cpu(), expect_append(case, kr, vr, ql, kl))


def test_append_one_row_each_and_strides():
    """One new token of each sequence (no boundaries), rows laid out head by head."""
    kl = [1, 0, 16, 17, 500]
    case = PoolCase(kl, 4, 64, 16)
    g = torch.Generator().manual_seed(4)
    kr, vr = torch.randn((2, 4, 5, 64), generator=g).unbind(0)  # [heads][rows][dim]
    k, v, lens, table = case.device()
    B.aio_page_append(kr.cuda().transpose(0, 1), vr.cuda().transpose(0, 1), k, v, lens, table)
    want = expect_append(case, kr.transpose(0, 1), vr.transpose(0, 1), [1] * 5, kl)
    assert same_bits(torch.stack((k, v)).cpu(), want)


def test_append_rounds_to_nearest_even():
    bits = torch.tensor([0x3f800000, 0x3f808000, 0x3f818000, 0x3f808001, 0x7f7fffff, 0x7f800000,
                         0xff800000 - (1 << 32), 0x7fc00001, 0x7f800001, 0x00000001, 0x80000000 - (1 << 32),
                         0x00008000, 0x00018000, 0x3f7fffff, 0x477fe000, 0x7f7f8000],
                        dtype=torch.int64).to(torch.int32).view(torch.float32)
    rowsv = bits.repeat(4).reshape(1, 1, 64)
    case = PoolCase([5], 1, 64, 16)
    k, v, lens, table = case.device()
    B.aio_page_append(rowsv.cuda(), (-rowsv).cuda(), k, v, lens, table)
    pg = int(case.table[0, 0])
    for got, src in ((k[pg, 0, 4], rowsv), (v[pg, 0, 4], -rowsv)):
        got, want = got.cpu(), src[0, 0].to(torch.bfloat16)
        nan = torch.isnan(want)
        assert torch.equal(torch.isnan(got), nan) and same_bits(got[~nan], want[~nan])


def test_append_stays_inside():
    """Rows before key 0, past the table, past max_len, of bad boundaries."""
    ql, kl = [12, 4, 5], [7, 64, 20]
    case = PoolCase([7, 40, 20], 2, 64, 16, width_more=0)
    g = torch.Generator().manual_seed(5)
    kr, vr = torch.randn((2, 21, 2, 64), generator=g).unbind(0)
    for lens in (kl, [7, 50, 1 << 30], [-3, 42, 20]):
        for max_len in (None, 18):
            k, v, _, table = case.device()
            ld = torch.tensor(lens, dtype=torch.int32, device="cuda")
            B.aio_page_append(kr.cuda(), vr.cuda(), k, v, ld, table, cu_q=cu(ql).cuda(),
                              max_len=max_len)
            want = expect_append(case, kr, vr, ql, lens, 1 << 30 if max_len is None else max_len)
            assert same_bits(torch.stack((k, v)).cpu(), want), (lens, max_len)
    for bad in ([0, 1 << 30, 5, 21], [-9, -5, -4, -3], [30, 40, 50, 60]):
        k, v, _, table = case.device()
        ld = torch.tensor(kl, dtype=torch.int32, device="cuda")
        B.aio_page_append(kr.cuda(), vr.cuda(), k, v, ld, table,
                          cu_q=torch.tensor(bad, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()


def test_append_through_a_narrow_view_of_a_table():
    """The columns of the table behind the view are not looked at."""
    case = PoolCase([30, 40], 1, 64, 16, width_more=0)
    g = torch.Generator().manual_seed(8)
    kr, vr = torch.randn((2, 60, 1, 64), generator=g).unbind(0)
    k, v, lens, table = case.device()
    B.aio_page_append(kr.cuda(), vr.cuda(), k, v, lens, table[:, :2], cu_q=cu([25, 35]).cuda(),
                      max_len=1000)
    want = expect_append(case, kr, vr, [25, 35], [30, 40], 32)
    assert same_bits(torch.stack((k, v)).cpu(), want)


def test_append_many_sequences():
    ql = [i % 3 for i in range(200)]
    kl = [q + i % 20 for i, q in enumerate(ql)]
    case = PoolCase(kl, 2, 64, 8)
    g = torch.Generator().manual_seed(6)
    kr, vr = torch.randn((2, sum(ql), 2, 64), generator=g).unbind(0)
    k, v, lens, table = case.device()
    B.aio_page_append(kr.cuda(), vr.cuda(), k, v, lens, table, cu_q=cu(ql).cuda())
    assert same_bits(torch.stack((k, v)).cpu(), expect_append(case, kr, vr, ql, kl))


# -------------------------------------------------------------------- copies

@pytest.mark.parametrize("planes,pages,shape,n", [
    (1, 2, (8,), 1), (2, 10, (2, 16, 64), 5), (48, 12, (8, 16, 128), 6), (3, 2000, (1, 8, 64), 1000),
    (2, 9, (1, 8, 64 * 33), 4)])
def test_copy(planes, pages, shape, n):
    g = torch.Generator(device="cuda").manual_seed(n)
    pool = torch.randn((planes, pages) + shape, generator=g, device="cuda").to(torch.bfloat16)
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(n)).numpy()
    src, dst = ids[:n], ids[n: 2 * n]
    want = pool.clone()
    want[:, torch.from_numpy(dst).cuda()] = pool[:, torch.from_numpy(src).cuda()]
    B.aio_page_copy(pool, src, dst)
    assert same_bits(pool, want)


def test_copy_one_source_to_several_and_strides():
    base = torch.randn((4, 6, 3, 40), device="cuda").to(torch.bfloat16)
    pool = base[:, :, :2]  # pages apart, the third part of each untouched
    want = base.clone()
    want[:, [1, 4, 5], :2] = base[:, [2, 2, 0], :2]
    B.aio_page_copy(pool, [2, 2, 0], [1, 4, 5])
    assert same_bits(base, want)
    with pytest.raises(B.AioError):
        B.aio_page_copy(pool, [2, 1], [1, 3])
    with pytest.raises(ValueError):
        B.aio_page_copy(base.transpose(2, 3), [0], [1])
    B.aio_page_copy(pool, [], [])
    assert same_bits(base, want)


def test_copy_in_a_graph():
    """The pairs travel with the captured launch; the host arrays may change."""
    pool = torch.randn((6, 8, 1, 16, 64), device="cuda").to(torch.bfloat16)
    src, dst = np.array([0, 1], np.int32), np.array([5, 6], np.int32)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.aio_page_copy(pool, src, dst)
    src[:], dst[:] = 7, 7
    for i in range(3):
        pool[:, :2].normal_()
        want = pool.clone()
        want[:, 5:7] = pool[:, :2]
        g.replay()
        torch.cuda.synchronize()
        assert same_bits(pool, want)
