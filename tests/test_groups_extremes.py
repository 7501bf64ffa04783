"""fp32 operands at the ends of their range: an infinite one reaches its own results alone, in parts and as it is,
and small ones keep the bits that their parts hold."""
import math

import pytest
import torch

from paper_2304_09590_amd import pnn
from tests.test_groups import F32, Case, steps

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("n,in_parts", [(30, False), (400, True)])
def test_an_infinite_operand_stays_in_its_row(n, in_parts):
    c = Case(n, 1, 4, 40, 24, F32)
    assert (n // 4 > 16) == in_parts
    row = int(torch.nonzero(c.kept)[0])
    e = int(c.ids[row, 0])
    x, dy = c.x.clone(), c.dy.clone()
    x[row, 5] = dy[row, 7] = math.inf
    for bad, good, w in ((pnn.grouped_forward(c.groups, x, c.w), pnn.grouped_forward(c.groups, c.x, c.w), c.w[e, :, 5]),
                         (pnn.grouped_backward_input(c.groups, dy, c.w), pnn.grouped_backward_input(c.groups, c.dy, c.w), c.w[e, 7])):
        assert (w != 0).all()
        assert torch.isnan(bad[row]).all() if in_parts else torch.equal(bad[row], w * math.inf)
        bad[row] = good[row]
        assert torch.equal(bad, good)
    dw, db = pnn.grouped_backward_weights(c.groups, dy, x)  # always in parts
    want, bwant = pnn.grouped_backward_weights(c.groups, c.dy, c.x)
    assert torch.isnan(dw[e, 7]).all() and torch.isnan(dw[e, :, 5]).all() and not torch.isfinite(db[e, 7])
    dw[e, 7], dw[e, :, 5], db[e, 7] = want[e, 7], want[e, :, 5], bwant[e, 7]
    assert torch.equal(dw, want) and torch.equal(db, bwant)


@gpu
@pytest.mark.parametrize("n", [30, 400])
@pytest.mark.parametrize("power", [-60, -100, -109, -115, -122])
def test_small_operands(n, power):
    """The third part of x ends at 2^-133: each value is off by half of that at most, beside the roundings of a sum."""
    c = Case(n, 1, 4, 40, 24, F32)
    g = torch.Generator().manual_seed(3)
    c.x = ((torch.rand(n, 40, generator=g) + 0.5) * 2.0 ** power).cuda()
    c.w = (torch.rand(4, 24, 40, generator=g) + 0.5).cuda()
    want, size = c.forward(None, 0.0)
    got = pnn.grouped_forward(c.groups, c.x, c.w).double()
    # (x in three roundings to bf16, the last at a step of 2^-133; w below 1.5, 40 of them; fp32's subnormals)
    tol = steps(40) * 2.0 ** -24 * size + 40 * 1.5 * 2.0 ** -134 + 2.0 ** -149
    assert ((got - want).abs() <= tol).all()
