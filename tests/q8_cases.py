"""Pools of 8-bit pages and of sequences that share prefixes, and a plain quantisation, for
the tests of the operators over them (CPU)."""
from __future__ import annotations

import math

import numpy as np
import torch

from tests.paged_cases import PoolCase


def quantise64(x):
    """(codes int8 [..., d], bytes uint8 [...]) of rows of any float type: b is the least of
    8 .. 248 for which the largest magnitude over 2^(b - 127), rounded to an integer (ties to
    even), is at most 127."""
    a = x.double().numpy()
    finite = np.isfinite(a).all(-1)
    a = np.where(finite[..., None], a, 0.0)
    top = np.abs(a).max(-1)
    b = np.full(top.shape, 248)
    for t in range(247, 7, -1):
        b = np.where(np.rint(np.ldexp(top, 127 - t)) <= 127, t, b)
    codes = np.clip(np.rint(np.ldexp(a, (127 - b)[..., None])), -127, 127)
    b = np.where(finite, b, 255)
    return torch.from_numpy(codes.astype(np.int8)), torch.from_numpy(b.astype(np.uint8))


def values(codes, exps):
    """The bf16 that codes and bytes stand for (exactly)."""
    scale = torch.from_numpy(np.ldexp(1.0, exps.numpy().astype(np.int64) - 127))
    scale = torch.where(exps == 255, torch.full_like(scale, math.nan), scale)
    v = codes.double() * scale[..., None]
    out = v.to(torch.bfloat16)
    assert torch.equal(out.double().nan_to_num(), v.nan_to_num())
    return out


class Q8Pool:
    """The pages of a PoolCase in 8 bits.  What no key occupies stands for infinities and NaN.
    ``case`` then holds what the codes stand for."""

    def __init__(self, case: PoolCase, layout="plain", seed=0):
        g = torch.Generator().manual_seed(seed)
        P, H, S, D = case.k.shape
        self.case, self.layout, self.shape = case, layout, (P, H, S, D)
        size = -(-H * S * (D + 1) // 16) * 16  # (pages lie whole numbers of 16 bytes apart)
        if layout == "plain":
            self.buffer = torch.zeros((2, P, size), dtype=torch.uint8)
        else:  # codes and bytes of K and V of a page beside one another
            self.buffer = torch.zeros((P, 2, size), dtype=torch.uint8)
        k, v, ke, ve = self.views(self.buffer)
        for codes, exps, pages in ((k, ke, case.k), (v, ve, case.v)):
            c, e = quantise64(pages.contiguous())
            free = torch.isnan(pages.float()).all(-1)
            junk = torch.randint(-128, 128, c.shape, generator=g).to(torch.int8)
            codes.copy_(torch.where(free[..., None], junk, c))
            exps.copy_(torch.where(free, torch.full_like(e, 255), e))
        for i in range(len(case.keys)):
            case.keys[i] = values(*quantise64(case.keys[i]))
            case.values[i] = values(*quantise64(case.values[i]))

    def views(self, buf):
        """(k, v, k_exp, v_exp) of a buffer like self.buffer."""
        P, H, S, D = self.shape
        out = []
        for w in range(2):
            part = buf[w] if self.layout == "plain" else buf[:, w]
            rows = H * S * D
            step = part.stride(0)
            out.append((part[:, :rows].view(torch.int8).as_strided(
                (P, H, S, D), (step, S * D, D, 1)),
                part[:, rows:].as_strided((P, H, S), (step, S, 1))))
        (k, ke), (v, ve) = out
        return k, v, ke, ve

    def device(self, dev="cuda"):
        """k, v, k_exp, v_exp, lens, table"""
        self.on = self.buffer.to(dev)
        return (*self.views(self.on), self.case.lens.to(dev), self.case.table.to(dev))


def group_case(k_len, groups, Hkv, hd, page, seed=0, holes=(), copied=False):
    """A PoolCase whose sequences first .. last - 1 of each (first, last, prefix) of groups begin
    with the same keys, in the first one's pages as far as pages are full (copied: in pages of
    their own)."""
    case = PoolCase(k_len, Hkv, hd, page, seed=seed, holes=holes)
    for first, last, prefix in groups:
        for i in range(first + 1, last):
            n = min(prefix, k_len[i], k_len[first])
            case.keys[i][:n] = case.keys[first][:n]
            case.values[i][:n] = case.values[first][:n]
            case.visible[i][:n] = case.visible[first][:n]
            for j in range(-(-n // page)):
                m = min(page, n - j * page)
                src, dst = int(case.table[first, j]), int(case.table[i, j])
                if m == page and not copied:
                    case.table[i, j] = src
                elif (first, j) in holes:
                    case.table[i, j] = -7
                else:
                    case.k[dst, :, :m] = case.k[src, :, :m]
                    case.v[dst, :, :m] = case.v[src, :, :m]
    return case
