"""Plain 64-bit evaluations of the operators over several sequences, on the
CPU, and the tolerances their tests use.

Attention.  With scores s_j = scale q.k_j (exact bf16 keys), weights p_j and A =
sum_j p_j |v_j|:
  * fp32 queries: a score is a sum of 3 hd products of exact terms.  Rounding
    errors of at most u = 2^-24 of the partial sums, which are at most B = scale
    sum_i |q_i k_ij|, are independent: their sum passes 4 sqrt(3 hd) u B for
    one score in 10^3 at most, 8 sqrt(3 hd) u B practically never.  The exponent's argument rounds
    once more (u |s| log2 e) and exp2 is off by at most 2^-22.  A weight is off by d = the
    sum of these, relatively, a normalised output by at most 2 d A, plus the sums
    over the keys (blocks of 32 to 64 in fp32: another 2^-20 A).
  * bf16: each weight is rounded to bf16 (at most 2^-8 of itself), each output
    too: 2^-8 (A + |out|) on top.
  * on average errors of fp32 queries cancel: an output's 2-norm is off by the
    rms error of a score, sqrt(3 hd) u |s|_rms, a few 1e-7; 4e-6 leaves room
    for the exponentials.
  * lse: d, plus the rounding of the result.
"""
from __future__ import annotations

import math

import numpy as np
import torch

U = 2.0 ** -24


def attention64(q, keys, values, q_len, k_len, visible=None, scale=None):
    """q [rows, H, hd]; keys, values: per sequence [k_len, Hkv, hd]; visible: per
    sequence a bool [k_len] of keys that are there.  Returns (out, lse, tol, lse_tol)
    in 64 bits for the rows of the sequences, in order.  Invisible keys and values take no part,
    whatever they hold."""
    rows, H, hd = q.shape
    scale = hd ** -0.5 if scale is None else scale
    out = torch.zeros((rows, H, hd), dtype=torch.float64)
    lse = torch.full((rows, H), -math.inf, dtype=torch.float64)
    tol = torch.zeros((rows, H, hd), dtype=torch.float64)
    ltol = torch.zeros((rows, H), dtype=torch.float64)
    bf16 = q.dtype == torch.bfloat16
    q64 = q.double()
    r0 = 0
    for i, (nq, nk) in enumerate(zip(q_len, k_len)):
        G = H // keys[i].shape[1]
        for r in range(nq):
            last = nk - nq + r
            at = torch.arange(last + 1) if last >= 0 else torch.arange(0)
            if visible is not None:
                at = at[visible[i][at]]
            if len(at) == 0:
                continue
            k = keys[i][at].double().repeat_interleave(G, dim=1)   # [t, H, hd]
            v = values[i][at].double().repeat_interleave(G, dim=1)
            prod = q64[r0 + r][None] * k
            s = scale * prod.sum(-1)
            B = scale * prod.abs().sum(-1)
            p = torch.softmax(s, dim=0)
            o = (p[..., None] * v).sum(0)
            A = (p[..., None] * v.abs()).sum(0)
            d = (8 * math.sqrt(3 * hd) * U * B + 1.5 * U * s.abs()).amax(0) + 2.0 ** -22
            out[r0 + r], lse[r0 + r] = o, torch.logsumexp(s, dim=0)
            tol[r0 + r] = 2 * d[:, None] * A + 2.0 ** -20 * A
            if bf16:
                tol[r0 + r] += 2.0 ** -8 * (A + o.abs()) * (1 + 2.0 ** -7)
            ltol[r0 + r] = d + 2.0 ** -22 * (1 + lse[r0 + r].abs())
        r0 += nq
    return out, lse, tol, ltol


def check_attention(got, lse, ref, what=""):
    out, l64, tol, ltol = ref
    n = out.shape[0]
    g = got[:n].double().cpu()
    err = (g - out).abs()
    bad = ~(err <= tol)
    bad &= ~(torch.isnan(g) & torch.isnan(out))
    assert not bad.any(), "%s: %d outputs off, worst %.3g of its tolerance" % (
        what, int(bad.sum()), float((err / tol.clamp_min(1e-30)).nan_to_num(nan=1e9).max()))
    if got.dtype == torch.float32 and torch.isfinite(out).all() and out.norm() > 0:
        rel = float((g - out).norm() / out.norm())
        assert rel <= 4e-6, (what, rel)
    if lse is not None:
        l = lse[:n].double().cpu()
        same = (l == l64) | (torch.isnan(l) & torch.isnan(l64))
        assert ((l - l64).abs().le(ltol) | same).all(), what


def logprobs64(x, targets, top):
    """(logprob, entropy, ids, top_logprobs, lp_tol, ent_tol) of fp32/bf16 rows.

    Tolerances.  With d = x - m, W = sum p |d|, W2 = sum p d^2: a term e^d is
    off by 2^-23 of itself (the exponential) and |d| (2^-24 + 2^-25) (the rounded
    product d log2 e, the rounded constant), and d by 2^-24 |d|; so log z is off
    by at most 2^-23 + 2^-22 W.  The terms of the weighted sum are off alike and by the
    rounding of up to 32 additions: 2^-23 W + 2^-22 W2 + 2^-19 W.  A result is
    rounded once, 2^-24 of itself."""
    x = x.double()
    m = x.amax(-1, keepdim=True)
    # against the maximum, not against the log-sum-exp itself: next to logits of
    # 3e38 the 64-bit sum m + log z drops log z
    logz = torch.log(torch.exp(x - m).sum(-1))
    y = (x - m) - logz[:, None]
    p = y.exp()
    ent = -torch.where(p > 0, p * y, torch.zeros_like(y)).sum(-1)
    ent = torch.where(torch.isfinite(logz), ent, torch.full_like(ent, math.nan))
    d = torch.where(p > 0, x - m, torch.zeros_like(y))
    W, W2 = (p * d.abs()).sum(-1), (p * d * d).sum(-1)
    lp_tol = 2.0 ** -23 + 2.0 ** -22 * W
    ent_tol = lp_tol + 2.0 ** -18 * W + 2.0 ** -22 * W2
    order = torch.from_numpy(np.argsort(
        np.where(np.isnan(x.numpy()), -math.inf, -x.numpy()), axis=-1, kind="stable"))
    # NaN first, in index order (argsort puts -inf first; real +Inf come after NaN)
    ids = []
    for r in range(x.shape[0]):
        nan = torch.isnan(x[r])
        o = order[r]
        ids.append(torch.cat((torch.nonzero(nan).flatten(), o[~nan[o]]))[:top])
    ids = torch.stack(ids) if x.shape[0] else torch.zeros((0, top), dtype=torch.int64)
    lp = None
    if targets is not None:
        ok = (targets >= 0) & (targets < x.shape[1])
        lp = y.gather(1, targets.clamp(0, x.shape[1] - 1).long()[:, None])[:, 0]
        lp = torch.where(ok, lp, torch.full_like(lp, math.nan))
    return lp, ent, ids, y.gather(1, ids), lp_tol, ent_tol


def close(got, want, tol):
    got = got.double().cpu()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    ok = same | ((got - want).abs() <= tol)
    assert ok.all(), (got[~ok][:4], want[~ok][:4])


class PoolCase:
    """Sequences of given lengths in shuffled pages; everything that no key of
    theirs occupies is NaN.  holes: (sequence, page index) pairs whose table entry
    is no page."""

    def __init__(self, k_len, Hkv, hd, page, seed=0, holes=(), layout="plain", spare=2,
                 width_more=1, garbage=(-1, 1 << 30, -(1 << 31), 7777)):
        g = torch.Generator().manual_seed(seed)
        n = len(k_len)
        counts = [-(-k // page) for k in k_len]
        n_pages = sum(counts) + spare
        width = max(counts + [0]) + width_more
        perm = torch.randperm(n_pages, generator=g).tolist()
        self.k_len, self.page, self.n_pages = list(k_len), page, n_pages
        nan = float("nan")
        if layout == "plain":
            pool = torch.full((2, n_pages, Hkv, page, hd), nan, dtype=torch.bfloat16)
            self.k, self.v = pool[0], pool[1]
        else:  # K and V of a page beside one another, a page's heads padded
            pool = torch.full((n_pages, 2, Hkv, page + 1, hd), nan, dtype=torch.bfloat16)
            self.k, self.v = pool[:, 0, :, :page], pool[:, 1, :, :page]
        self.pool = pool
        self.layout = layout
        # what lies behind a row's last page is anything
        self.table = torch.tensor([[garbage[(i + j) % len(garbage)] for j in range(width)]
                                   for i in range(n)], dtype=torch.int32).reshape(n, width)
        self.keys, self.values, self.visible = [], [], []
        at = 0
        for i, (kl, c) in enumerate(zip(k_len, counts)):
            k = torch.randn((kl, Hkv, hd), generator=g).to(torch.bfloat16)
            v = torch.randn((kl, Hkv, hd), generator=g).to(torch.bfloat16)
            vis = torch.ones(kl, dtype=torch.bool)
            for j in range(c):
                pg = perm[at + j]
                self.table[i, j] = pg
                m = min(page, kl - j * page)
                self.k[pg, :, :m] = k[j * page: j * page + m].transpose(0, 1)
                self.v[pg, :, :m] = v[j * page: j * page + m].transpose(0, 1)
                if (i, j) in holes:
                    self.table[i, j] = (-1, n_pages, 1 << 30)[j % 3]
                    vis[j * page: j * page + m] = False
            at += c
            self.keys.append(k)
            self.values.append(v)
            self.visible.append(vis)
        self.lens = torch.tensor(list(k_len), dtype=torch.int32)

    def device(self, dev="cuda"):
        pool = self.pool.to(dev)
        if self.layout == "plain":
            k, v = pool[0], pool[1]
        else:
            k, v = pool[:, 0, :, : self.page], pool[:, 1, :, : self.page]
        return k, v, self.lens.to(dev), self.table.to(dev)


def cu(sizes):
    return torch.tensor(np.concatenate(([0], np.cumsum(sizes))), dtype=torch.int32)
