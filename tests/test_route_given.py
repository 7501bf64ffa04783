"""Gradients of scores at ids of the caller's: many rows a wave, networks that stand twice, choices far below a row's largest."""
import pytest
import torch

from paper_2304_09590_amd import pnn
from tests.test_route import case, near, reference

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,K,k", [(70000, 10, 3), (40000, 60, 5), (20000, 200, 20), (9000, 200, 4), (9000, 450, 3), (5000, 1000, 33)])
def test_rows_after_each_other_on_the_same_lanes(n, K, k, dtype):
    """A wave's rows share places in LDS: what a row's choices leave there is gone when the next one's come, whichever lanes wrote it."""
    s, dgates = case(n, K, k, dtype, seed=n)
    ids = torch.randint(-1, K + 1, (n, k), generator=torch.Generator().manual_seed(K), dtype=torch.int32)
    ids[::3, 1] = ids[::3, 0]
    ids[1::7] = ids[1::7, :1]
    ids[2::5] = (torch.arange(n)[2::5, None] // 5 + torch.arange(k)).to(torch.int32) % K  # (a network moves from lane to lane)
    ids = ids.cuda()
    for normalize in (False, True):
        near(pnn.route_grad(s, ids, None, dgates, normalize=normalize), *reference(s, k, normalize, dgates, 0.0, ids)[4], dtype=dtype)
