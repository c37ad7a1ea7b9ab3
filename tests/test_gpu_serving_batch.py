"""The operators of a serving batch together, as a serving loop runs them: requests forked
from cached templates, their query and key rows normed and rotated, rows appended to pages of 8
bits or bf16, attention behind the shared templates; several turns, against a plain evaluation of
every request by itself."""
import numpy as np
import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import attention64, check_attention, cu
from tests.q8_cases import quantise64, values
from tests.test_gpu_qk_norm_rope import norm64

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
H, HKV, HD, PAGE = 8, 2, 64, 16


class Server:
    """One layer's cache, in 8 bits or bf16, and its requests."""

    def __init__(self, q8, dtype, n_pages=160, max_seqs=24):
        self.q8, self.dtype = q8, dtype
        self.pages = B.Pages(n_pages, PAGE, max_seqs)
        rows = HKV * PAGE * HD
        if q8:  # codes and bytes of a page beside one another: a page is one copy
            self.pool = torch.zeros((2, n_pages, HKV * PAGE * (HD + 1)), dtype=torch.uint8,
                                    device="cuda")
            kv = [(self.pool[w, :, :rows].view(torch.int8).unflatten(1, (HKV, PAGE, HD)),
                   self.pool[w, :, rows:].unflatten(1, (HKV, PAGE))) for w in range(2)]
            self.kv = [kv[0][0], kv[1][0], kv[0][1], kv[1][1]]
        else:
            self.pool = torch.zeros((2, n_pages, HKV, PAGE, HD), dtype=BF16, device="cuda")
            self.kv = [self.pool[0], self.pool[1]]
        g = torch.Generator().manual_seed(11)
        self.w = [(1 + 0.1 * torch.randn(HD, generator=g)).to(BF16) for _ in range(2)]
        self.keys, self.values, self.gen = {}, {}, g

    def template(self, n):
        """A sequence of n positions; no query is asked of it."""
        s = self.pages.open()
        self.keys[s] = self.values[s] = torch.empty((0, HKV, HD), dtype=BF16)
        self.turn([s], [n])
        return s

    def fork(self, s):
        c = self.pages.fork(s)
        self.keys[c], self.values[c] = self.keys[s], self.values[s]
        return c

    def turn(self, seqs, counts, groups=None, idle=0):
        """counts[i] new rows of sequence i: (queries as given, attention's outputs and lse)."""
        src, dst, pos = [], [], []
        for s, n in zip(seqs, counts):
            at = self.pages.length(s)
            a, b = self.pages.extend(s, n)
            src += a
            dst += b
            pos += range(at, at + n)
        if src:
            B.aio_page_copy(self.pool.view(2, self.pool.shape[1], -1), src, dst)
        lens, table = self.pages.rows(seqs, 40)
        lens = np.concatenate((lens, np.zeros(idle, np.int32)))  # idle places of a padded batch
        table = np.concatenate((table, np.full((idle, 40), -1, np.int32)))
        lens, table = torch.from_numpy(lens).cuda(), torch.from_numpy(table).cuda()
        n = len(pos) + idle
        qkv = torch.randn((n, H + 2 * HKV, HD), generator=self.gen).to(self.dtype)
        pos = torch.tensor(pos + [0] * idle, dtype=torch.int32)
        d = qkv.cuda()
        q, k, v = d[:, :H], d[:, H: H + HKV], d[:, H + HKV:]
        B.aio_qk_norm_rope(q, k, pos.cuda(), q, k, self.w[0].cuda(), self.w[1].cuda())
        one = all(c == 1 for c in counts)
        c = None if one else cu(list(counts) + [0] * idle).cuda()
        rows = (k, v)
        if not one:
            rows = (k[: n - idle], v[: n - idle])
        append = B.aio_q8_append if self.q8 else B.aio_page_append
        if one and idle:  # (an idle place appends before key 0, which is nowhere)
            append(*rows, *self.kv, lens, table)
        else:
            append(*rows, *self.kv, lens, table, cu_q=c)
        # what the rows were, on the CPU, from the rotated rows as the call left them
        r = 0
        for s, m in zip(seqs, counts):
            kr, vr = k[r: r + m].cpu(), v[r: r + m].cpu()
            stand = (lambda t: values(*quantise64(t))) if self.q8 else (lambda t: t.to(BF16))
            self.keys[s] = torch.cat((self.keys[s], stand(kr)))
            self.values[s] = torch.cat((self.values[s], stand(vr)))
            r += m
        want, tol = norm64(qkv[:, :H], pos, self.w[0], 1e-5, 1e4)
        assert ((q.double().cpu() - want).abs() <= tol).all()
        if groups is None:
            return None
        out = torch.empty((n if one else n - idle, H, HD), dtype=self.dtype, device="cuda")
        lse = torch.empty(out.shape[:2], device="cuda")
        first, prefix = groups
        f = B.aio_q8_prefix_attention if self.q8 else B.aio_prefix_attention
        f(q[: out.shape[0]], *self.kv, lens, table,
          torch.tensor(first, dtype=torch.int32, device="cuda"),
          torch.tensor(prefix, dtype=torch.int32, device="cuda"), out, cu_q=c, lse=lse,
          max_len=int(lens.max()), max_prefix=max(prefix))
        m = sum(counts)
        ref = attention64(q[:m].cpu(), [self.keys[s] for s in seqs],
                          [self.values[s] for s in seqs], counts,
                          [self.pages.length(s) for s in seqs])
        check_attention(out[:m], lse[:m], ref)
        if one and idle:
            assert (out[m:] == 0).all() and (lse[m:] == -float("inf")).all()
        return out


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("q8", [True, False])
def test_requests_behind_two_templates(q8, dtype):
    s = Server(q8, dtype)
    a, b = s.template(203), s.template(130)
    seqs = [s.fork(a) for _ in range(13)] + [s.fork(b) for _ in range(4)]
    groups = ([0, 13, 17], [203, 130])
    # the requests' own prompts, several tokens, a padded place among the steps
    s.turn(seqs, [3 + 5 * (i % 4) for i in range(17)], groups)
    for step in range(3):
        s.turn(seqs, [1] * 17, ([0, 13, 17], [203, 130]), idle=step)
    # a rejected draft is cut off, a request leaves, one goes on with a long turn
    s.pages.truncate(seqs[2], 205)
    s.keys[seqs[2]], s.values[seqs[2]] = s.keys[seqs[2]][:205], s.values[seqs[2]][:205]
    s.pages.close(seqs[5])
    seqs = seqs[:5] + seqs[6:]
    s.turn(seqs, [1] * 10 + [70] + [2] * 5, ([0, 12, 16], [203, 130]))
    s.turn(seqs, [1] * 16, ([0, 12, 16], [203, 130]))
