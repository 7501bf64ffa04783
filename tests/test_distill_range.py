"""The distillation loss and its gradient where a scaled maximum is large: masks by finite constants, far-off and
single large logits, small temperatures, running maxima that grow past the point from which differences are
taken before they are scaled."""
import math

import pytest
import torch

from paper_2304_09590_amd import pnn
from tests.test_distill import BF16, F32, case, verify

gpu = pytest.mark.gpu
WIDTHS = [(8, 12, 4), (8, 100, 20), (8, 700, 40), (8, 3000, 9), (8, 9000, 9)]  # 16 lanes, a wave, a workgroup, parts of a row
TEMPERATURES = [1e-6, 1e-4, 0.5, 1.0, 2.0, 8.0, 1e6]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("n,v,k", WIDTHS)
def test_rows_alike_and_single_large_logits(n, v, k, temperature, dtype):
    """All classes at a constant of any size, or all but one: what the loss is of zeros, or of one class alone."""
    z, idx, t, y, g = case(n, v, k, dtype, seed=17)
    for r, value in enumerate((-1e4, -1e10, -1e20, -1e30, 1e10, 1e30)):
        z[r] = value
    z[6, 5] = 1e10                             # (a small logit among millions: in the sum it has no weight)
    z[7, v - 1] = 1e30
    idx[6, 0], y[6] = 5, 5
    idx[7, 0], y[7] = v - 1, v - 1
    idx[6:, 1:] = -1                           # (the one class is all that the teacher answers)
    loss, dz = verify(z, idx, t, y, g, temperature, 0.25)
    assert torch.isfinite(loss).all() and torch.isfinite(dz).all() and (loss[:6] > 0).all()
    loss, dz = verify(z, idx, t, None, g, temperature, 0.0)
    assert (loss[6:] == 0).all() and (dz[6:] == 0).all()
    verify(z, idx, t, y, g, temperature, 1.0)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("n,v,k", WIDTHS)
def test_masks_by_constants(n, v, k, temperature, dtype):
    """Half of the classes at a constant far below the others, and logits of the size of thousands."""
    z, idx, t, y, g = case(n, v, k, dtype, seed=19)
    masked = torch.rand(n, v, generator=torch.Generator().manual_seed(2)).cuda() < 0.5
    masked[torch.arange(n).cuda()[:, None], idx.long()] = False
    masked[torch.arange(n).cuda(), y.long()] = False
    for value in (-1e5, -1e10, -1e30):
        verify(torch.where(masked, torch.tensor(value, dtype=dtype, device="cuda"), z), idx, t, y, g, temperature, 0.25)
    verify(z * 2000, idx, t, y, g, temperature, 0.25)


@gpu
@pytest.mark.parametrize("temperature,alpha", [(1.0, 0.25), (2.0, 0.25), (3.0, 0.25), (0.5, 0.0), (2.0, 1.0)])
@pytest.mark.parametrize("n,v,k", WIDTHS)
def test_maxima_that_grow_past_the_switch(n, v, k, temperature, alpha):
    """Neighbouring fp32 values about where a scaled maximum is 2^20, in both signs, rising and falling along the row."""
    _, idx, t, y, g = case(n, v, k, F32, seed=21)
    scale = math.log2(math.e) * max(1.0 / temperature if alpha < 1 else 1.0, 1.0 if alpha > 0 else 0.0)
    middle = 2.0 ** 20 / scale
    gen = torch.Generator().manual_seed(4)
    d = torch.randint(-64, 65, (n, v), generator=gen).double() / 16
    d[:2] = d[:2].sort(1).values
    d[2:4] = d[2:4].sort(1, descending=True).values
    d[4:6] = d[4:6].sort(1).values / 8
    z = (d + middle).float()
    z[1::2] = (d[1::2] - middle).float()
    verify(z.cuda(), idx, t, y if alpha > 0 else None, g, temperature, alpha)
