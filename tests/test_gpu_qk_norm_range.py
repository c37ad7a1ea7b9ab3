"""The norm of rows whose squares, eps, or the sum of both lie at the ends of a float's range,
with the tolerance of the other norms: a mean square is a sum of rounded squares only where these
are normal numbers, so the operator has to scale."""
import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.test_gpu_qk_norm_rope import BF16, F32, check, make

pytestmark = pytest.mark.gpu


def size_of(x, size):
    """Rows of standard deviation ``size``; one has a single element, one none."""
    x = (x.double() * size).float()
    x[3, 0, 5:] = 0
    x[4] = 0
    return x


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size,eps", [
    # squares past the largest float beside an eps that counts, and an eps that alone brings them there
    (1e19, 1e38), (1e19, 3e38), (1e18, 3e38), (3e18, 3e38), (1e18, 3.4e38), (1e25, 3e38),
    # squares and eps below the smallest normal float
    (1e-20, 1e-42), (1e-21, 1e-43), (1e-22, 1.5e-45), (1e-19, 1.5e-45), (1e-25, 1e-45), (1e-30, 1e-40),
    (1e-17, 1e-33), (1e-13, 1e-27), (1e-14, 1e-45), (1e-13, 1e-45),
])
def test_ends_of_the_range(size, eps, dtype, hd):
    qkv, pos, w = make(6, 2, 1, hd, F32)
    qkv = size_of(qkv, size).to(dtype)
    e = float(torch.tensor(eps, dtype=F32))
    assert 0 < e < float("inf")
    d = qkv.cuda()
    qo, ko = torch.empty_like(d[:, :2]), torch.empty_like(d[:, 2:3])
    B.aio_qk_norm_rope(d[:, :2], d[:, 2:3], pos.cuda(), qo, ko, q_weight=w[0].cuda(), eps=eps)
    check(qo, qkv[:, :2], pos, w[0], e)
    check(ko, qkv[:, 2:3], pos, None, e)
    assert (qo[4] == 0).all() and (ko[4] == 0).all()
