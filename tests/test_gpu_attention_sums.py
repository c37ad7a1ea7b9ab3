"""Attention over many keys that are all alike: a sum of equal terms rounds the same way
at each addition, so one long chain drifts where a short context or scores that differ
show nothing.

The queries are one unit vector and each key a multiple b of it, so scores are exact.  In
units of 2^-24 of the value (b is at most 4.1): a weight is off by 2 b (the scale's factor
log2 e and the exponent's argument round) and 4 (exp2): 16 at most.  A sum of
weights: 16 for the 32 additions within a block, 24 with the carries and the joins of
lanes, waves and splits: 40 together.  A value that one key alone has: its weight, the sum and the
division, 64.  A value that all keys have: 96 (one token) or 384 (prompts) matrix
instructions that add to one sum before it is carried, each off by a unit in the last
place, 2, of what is there then, half the sum on average.  The log-sum-exp is below 20: a
logarithm off by two units in the last place of 16 (32), the reference's product and sum (32)."""
import math

import pytest
import torch

from paper_2604_09752_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def inputs(n, hd, first, n_first, rest):
    """Keys: n_first of score `first`, then `rest`; values: 1 in dimension 1, in
    dimension 0 only the last key's."""
    k = torch.zeros((n, 1, hd), dtype=torch.bfloat16)
    k[:n_first, 0, 0], k[n_first:, 0, 0] = first, rest
    v = torch.zeros_like(k)
    v[:, 0, 1] = 1
    v[n - 1, 0, 0] = 1
    return k, v


def check(out, lse, n, first, n_first, rest, chain, bf16, what):
    z = n_first * math.exp(first) + (n - n_first) * math.exp(rest)
    own = math.exp(rest) / z
    more = 2.0 ** -8 + 2.0 ** -7 if bf16 else 0.0  # the weight and the output in bf16
    assert abs(lse - math.log(z)) <= 104 * U, (what, lse - math.log(z))
    assert abs(out[0] / own - 1) <= 64 * U + more, (what, out[0] / own - 1)
    assert abs(out[1] - 1) <= (chain + 40) * U + more, (what, out[1] - 1)


SCORES = [(0.0, 64, 4.09375), (0.0, 64, 2.0), (0.0, 64, 1.296875), (0.296875, 1, 0.0),
          (4.09375, 1, 0.0), (1.5, 1, 0.0)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("seqs", [1, 1024])  # the keys split over workgroups, and not
@pytest.mark.parametrize("n", [4096, 32768, 131072])
def test_one_token(n, seqs, hd, dtype):
    for first, n_first, rest in SCORES:
        k, v = inputs(n, hd, first, n_first, rest)
        k, v = (t.reshape(n // 64, 64, 1, hd).transpose(1, 2).contiguous().cuda() for t in (k, v))
        table = torch.arange(n // 64, dtype=torch.int32, device="cuda")[None].repeat(seqs, 1)
        lens = torch.full((seqs,), n, dtype=torch.int32, device="cuda")
        q = torch.zeros((seqs, 1, hd), dtype=dtype, device="cuda")
        q[:, :, 0] = 1
        out, lse = torch.empty_like(q), torch.empty((seqs, 1), device="cuda")
        B.aio_paged_attention(q, k, v, lens, table, out, lse=lse, scale=1.0, max_len=n)
        for i in {0, seqs - 1}:
            check(out[i, 0].tolist(), lse[i, 0].item(), n, first, n_first, rest, 96,
                  dtype == torch.bfloat16, (n, seqs, hd, first, rest))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows", [1, 65536])  # the keys split over workgroups, and not
@pytest.mark.parametrize("n", [4096, 32768, 131072])
def test_prompts(n, rows, hd, dtype):
    rows = min(rows, n)
    q = torch.zeros((rows, 1, hd), dtype=dtype, device="cuda")
    q[:, :, 0] = 1
    out, lse = torch.empty_like(q), torch.empty((rows, 1), device="cuda")
    cu_q, cu_k = (torch.tensor([0, t], dtype=torch.int32, device="cuda") for t in (rows, n))
    for first, n_first, rest in SCORES:
        k, v = inputs(n, hd, first, n_first, rest)
        B.aio_packed_attention(q, k.cuda(), v.cuda(), cu_q, cu_k, out, lse=lse, scale=1.0)
        check(out[-1, 0].tolist(), lse[-1, 0].item(), n, first, n_first, rest, 384,
              dtype == torch.bfloat16, (n, rows, hd, first, rest))
