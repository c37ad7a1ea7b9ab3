"""Prompt rows in tiles of 256 (bf16 queries, enough rows and heads): sampled rows and
heads against 64 bits, every row against fp32 queries of the same values, which take
tiles of 128."""
import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import PoolCase, attention64, check_attention, cu

pytestmark = pytest.mark.gpu

# heads, kv heads, head dimension, rows and keys per sequence, holes (sequence, page of 16),
# waves of a workgroup
CASES = {
    "three_hd64": (128, 16, 64, [1100, 1, 1003], [1100, 90, 1400], (), 8),
    "one_hd64": (128, 16, 64, [2048], [2300], (), 8),
    "one_hd128": (64, 8, 128, [4100], [4100], (), 8),
    "many_hd128": (32, 32, 128, [300] * 26 + [393], [300 + 17 * i for i in range(27)], (), 8),
    "group_of_3": (96, 32, 64, [2731], [2731], (), 8),
    "group_of_16": (128, 8, 64, [0, 2047, 7], [3, 2047, 7], (), 8),
    "holes": (64, 8, 128, [2100, 2000], [2100, 2500], ((0, 3), (0, 100), (1, 7), (1, 140)), 8),
    "before_the_first_key": (128, 16, 64, [2100], [1500], (), 8),
    "just_below": (128, 16, 64, [2045], [2045], (), 4),
}


def sampled(q, case, ql, heads):
    """The reference of some rows of some heads: (their indices, one reference a head)."""
    starts = cu(ql).tolist()
    at, keys, values, seen, vis = [], [], [], [], []
    for i, m in enumerate(ql):
        for r in sorted({0, 1, 31, 32, 255, 256, m // 2, m - 1}):
            if not 0 <= r < m or (m < 400 and r not in (0, m - 1)):
                continue
            n = max(case.k_len[i] - m + r + 1, 0)
            at.append(starts[i] + r)
            seen.append(n)
            keys.append(case.keys[i][:n])
            values.append(case.values[i][:n])
            vis.append(case.visible[i][:n])
    H, Hkv = q.shape[1], case.keys[0].shape[1]
    refs = []
    for h in heads:
        g = h // (H // Hkv)
        refs.append(attention64(q[at][:, h: h + 1], [k[:, g: g + 1] for k in keys],
                                [v[:, g: g + 1] for v in values], [1] * len(at), seen, vis))
    return at, refs


@pytest.mark.parametrize("name", list(CASES))
def test_tiles_of_256_rows(name):
    H, Hkv, hd, ql, kl, holes, _ = CASES[name]
    case = PoolCase(kl, Hkv, hd, 16, seed=len(name), holes=holes)
    n = sum(ql)
    q = torch.randn((n + 2, H, hd), generator=torch.Generator().manual_seed(n)).to(torch.bfloat16)
    heads = (0, H // Hkv - 1, H - 1)
    at, refs = sampled(q, case, ql, heads)
    k, v, lens, table = case.device()
    qd, qf, c = q.cuda(), q.float().cuda(), cu(ql).cuda()
    kp, vp = torch.cat(case.keys).cuda(), torch.cat(case.values).cuda()
    for form in ("pages", "packed"):
        if form == "packed" and holes:
            continue

        def attend(x):
            out, lse = torch.full_like(x, 9.0), torch.full(x.shape[:2], 9.0, device="cuda")
            if form == "pages":
                B.aio_paged_attention(x, k, v, lens, table, out, cu_q=c, lse=lse, max_len=max(kl))
            else:
                B.aio_packed_attention(x, kp, vp, c, cu(kl).cuda(), out, lse=lse)
            return out, lse

        out, lse = attend(qd)
        for h, ref in zip(heads, refs):
            check_attention(out[at][:, h: h + 1], lse[at][:, h: h + 1], ref, (name, form, h))
        assert (out[n:] == 9).all() and (lse[n:] == 9).all()
        of, lf = attend(qf)
        # each weight and each output rounds to bf16, 2^-8 of at most the largest value;
        # and the fp32 rows are off by far less than one such rounding more
        most = float(torch.cat(case.values).float().abs().max())
        assert (out[:n].float() - of[:n]).abs().max() <= 3 * 2.0 ** -8 * most, (name, form)
        # (both sum unrounded weights of equal scores, each off by at most 4 sqrt(3 hd)
        # 2^-24 sum |q k| / sqrt(hd), which is below 12 here)
        same = (lse == lf) | ((lse - lf).abs() <= 2.0 ** -13)
        assert same.all(), (name, form)


def test_later_values_that_are_not_finite():
    """Keys and values behind a row's own, in its last tile and in later ones."""
    H, Hkv, hd, n = 128, 16, 64, 2100
    case = PoolCase([n], Hkv, hd, 16)
    q = torch.randn((n, H, hd), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    clean, _ = run(q, case.keys[0], case.values[0])
    for at in (70, 1024, n - 25):
        keys, values = case.keys[0].clone(), case.values[0].clone()
        values[at, :, 7] = float("inf")
        keys[at + 5, :, 3] = float("nan")
        out, lse = run(q, keys, values)
        assert torch.equal(out[:at], clean[:at])
        assert not torch.isfinite(out[at:, :, 7]).any()
        keep = [d for d in range(hd) if d != 7]
        mid = (out[at: at + 5][:, :, keep].float() - clean[at: at + 5][:, :, keep].float()).abs()
        assert mid.max() <= 2.0 ** -7 * float(case.values[0].abs().max())
        assert torch.isnan(lse[at + 5:]).all() and torch.isfinite(lse[: at + 5]).all()


def run(q, keys, values):
    out, lse = torch.empty_like(q).cuda(), torch.empty(q.shape[:2], device="cuda")
    c = cu([q.shape[0]]).cuda()
    B.aio_packed_attention(q.cuda(), keys.cuda(), values.cuda(), c, c, out, lse=lse)
    return out, lse
