"""Weight gradients whose networks lie between each other's rows, and what overlaps."""
import pytest
import torch

from paper_2304_09590_amd import pnn
from tests.test_groups import BF16, F32, Case, backward_weights, groups_of

gpu = pytest.mark.gpu


@pytest.mark.parametrize("dw_net,dw_ld,overlap", [(40, 8, False), (39, 8, True), (8, 24, False), (9, 26, False), (8, 23, True), (7, 24, True),
                                                  (0, 24, True), (-8, 24, True), (12, 24, True), (1000, 24, False), (103, 24, True)])
def test_networks_that_overlap_are_refused(dw_net, dw_ld, overlap):
    """Three networks of 5 x 8; the call that passes this check stops at its missing workspace."""
    status = backward_weights(g=groups_of(n=5000), dw_net=dw_net, dw_ld=dw_ld)
    assert status == (pnn.PNN_EINVAL if overlap else pnn.PNN_ESHAPE)
    assert ("overlap" in pnn.lib().pnn_last_error(None).decode()) == overlap


@pytest.mark.parametrize("dw_net,dw_ld,overlap", [(40, 1 << 62, False), (1 << 61, 1 << 62, True), ((1 << 63) - 1, 1 << 62, True),
                                                  (1 << 62, 1 << 60, True), ((1 << 62) + 8, 1 << 60, False)])
def test_strides_near_the_end_of_64_bits(dw_net, dw_ld, overlap):
    test_networks_that_overlap_are_refused(dw_net, dw_ld, overlap)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,networks,inputs,outputs,pad", [(300, 5, 64, 128, 0), (5000, 2, 24, 40, 0), (3000, 3, 33, 17, 1), (4000, 3, 520, 264, 0)])
def test_networks_between_each_others_rows(n, networks, inputs, outputs, pad, dtype):
    """dw as [outputs][networks][inputs], with room that stays as it was."""
    c = Case(n, 1, networks, inputs, outputs, dtype, pad=pad)
    want, bwant = pnn.grouped_backward_weights(c.groups, c.dy, c.x)
    whole = torch.full((outputs + 2, networks, inputs + 5), 7.0, device="cuda")
    plain = whole.clone()
    view = whole[1:-1, :, 2:-3].permute(1, 0, 2)
    dw, db = pnn.grouped_backward_weights(c.groups, c.dy, c.x, dw=view)
    plain[1:-1, :, 2:-3] = want.permute(1, 0, 2)
    assert dw is view and torch.equal(whole, plain) and torch.equal(db, bwant)
