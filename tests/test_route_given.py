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


U = 2.0 ** -24


def among_the_chosen(s, ids, dgates):
    """The gradient through gates that are softmax among a row's ids, in 64 bits, and what it may be off by: an exponential of d by
    (3 |d| + 2) U, the sum by its terms' and a step for each addition, then a quotient and products."""
    K = s.shape[1]
    i = ids.cpu().long()
    kept = (i >= 0) & (i < K)
    at = torch.where(kept, i, 0)
    x = torch.where(kept, s.double().cpu().gather(1, at), -float("inf"))
    top = x.amax(1, keepdim=True)
    d = x - torch.where(torch.isfinite(top), top, 0.0)
    e = torch.exp(d)
    gates = e / torch.where(torch.isfinite(top), e.sum(1, keepdim=True), 1.0)
    dg = torch.where(kept, dgates.double().cpu(), 0.0)
    mix = (gates * dg).sum(1, keepdim=True)
    rel = torch.where(gates > 0, (3 * d.abs() + 8) * U, 0.0)
    rel = rel + (gates * rel).sum(1, keepdim=True) + 70 * U
    mixoff = (gates * dg.abs() * (rel + 40 * U)).sum(1, keepdim=True)
    off = gates * (rel * (dg - mix).abs() + mixoff + 8 * U * (dg.abs() + mix.abs()))
    want, size = torch.zeros(s.shape, dtype=torch.float64), torch.zeros(s.shape, dtype=torch.float64)
    return want.scatter_add(1, at, gates * (dg - mix)), size.scatter_add(1, at, off) + 1e-37


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,K,k", [(50, 3, 2), (9000, 16, 3), (9000, 200, 5), (200, 60, 9), (100, 500, 20), (60, 1000, 64)])
def test_gates_among_networks_far_below_the_largest(n, K, k, dtype):
    """A row's gates are among its chosen networks, however far others are above them."""
    s, dgates = case(n, K, k, dtype, seed=K, scale=1.0)
    s[:, 0] += torch.tensor([0.0, 80.0, 100.0, 150.0, 1e4, 1e30], device="cuda")[torch.arange(n, device="cuda") % 6].to(dtype)
    ids = torch.stack([torch.randperm(K - 1, generator=torch.Generator().manual_seed(r))[:k] + 1 for r in range(n)]).to(torch.int32)
    ids[1::8, 1:] = -1                        # one network: its gate is 1, whatever its score
    ids[3::8] = K                             # none
    s[5::8, 1] = -float("inf")
    s[6::8, 1:] = -float("inf")               # all chosen ones are masked
    s[7::8, 1:] -= 3e38                       # (the lowest ones)
    ids = ids.cuda()
    got = pnn.route_grad(s, ids, None, dgates, normalize=True)
    want, off = among_the_chosen(s, ids, dgates)
    assert (got[1::8] == 0).all() and (got[3::8] == 0).all() and (got[6::8] == 0).all()
    assert (want[4::12].abs().sum(1) > 1e-3).any()
    near(got, want, off, dtype=dtype)
    # the balance loss's share does not change with it
    counts, one = torch.ones(K + 1, dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda")
    alone = pnn.route_grad(s.float(), ids, counts, None, one, normalize=True).double().cpu()
    both = pnn.route_grad(s.float(), ids, counts, dgates, one, normalize=True)
    want, off = among_the_chosen(s.float(), ids, dgates)
    near(both, want + alone, off + U * (want + alone).abs() + 4 * U * want.abs())


@gpu
@pytest.mark.parametrize("n,K,k", [(9, 16, 16), (9000, 40, 33), (100, 200, 64), (5000, 500, 40), (64, 1000, 64)])
def test_gates_of_rows_with_a_wide_spread(n, K, k):
    """Scores whose differences are exact, down to 80 below the largest: a gate is off by its exponential's four half steps, the sum's and a
    quotient's, whatever its size."""
    g = torch.Generator().manual_seed(K)
    s = (torch.rand(n, K, generator=g) * 80 * 16).floor() / 16  # (11 bits)
    s[:, 0] = 80.0
    for normalize in (False, True):
        ids, gates, _, _ = pnn.route(s.cuda(), k, normalize=normalize)
        x = s.double().gather(1, ids.cpu().long())
        e = torch.exp(s.double() - 80)
        # (terms of the sum: 3 |d| + 2 each, far ones weigh little)
        rel = ((e * (3 * (80 - s.double()) + 2)).sum(1, keepdim=True) / e.sum(1, keepdim=True) + 40) * U
        want = torch.softmax(x, 1) if normalize else torch.exp(x - 80) / e.sum(1, keepdim=True)
        assert ((gates.double().cpu() - want).abs() <= want * (8 * U + rel) + 1e-37).all()
