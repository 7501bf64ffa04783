"""Products of codes with scales at the ends of fp32's range: what the formula gives within the range comes out, whichever way a row's and an
output's scale go."""
import numpy as np
import pytest
import torch

from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
MOST = float(np.finfo(np.float32).max)


def scales(size, powers, seed):
    g = np.random.default_rng(seed)
    return ((1 + g.random(size)) * np.exp2(g.choice(powers, size).astype(np.float64))).astype(np.float32)


# (pairs a network in the mean: at most two, tiles of 128 x 64, 256 x 256, 256 x 128)
SHAPES = [(3, 2, 9, 48, 33), (70, 2, 5, 80, 203), (4096, 1, 4, 64, 2049), (4096, 1, 16, 96, 3329)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("n,k,K,I,O", SHAPES)
def test_scales_from_one_end_to_the_other(n, k, K, I, O, bias, dtype):
    g = np.random.default_rng(n)
    x, w = g.integers(-127, 128, (n, I)).astype(np.int8), g.integers(-127, 128, (K, O, I)).astype(np.int8)
    w[:, :, 0], x[:, 0] = 127, 127
    xs, ws = scales((n,), [-126, -110, -91, -60, 0, 60, 91, 110, 120], 1), scales((K, O), [-126, -100, -50, 0, 50, 100, 120], 2)
    b = g.standard_normal((K, O)).astype(np.float32)
    ids = g.integers(0, K, (n, k)).astype(np.int32)

    def dev(a):
        return torch.from_numpy(a).cuda()

    y = pnn.grouped_forward_int8(pnn.group_rows(dev(ids), K), dev(x), dev(xs), dev(w), dev(ws), dev(b) if bias else None, out_dtype=dtype)
    got = y.double().cpu().numpy()
    e, r = ids.reshape(-1), np.arange(n * k) // k
    sums = np.empty((n * k, O))
    for i in range(K):
        at = np.nonzero(e == i)[0]
        sums[at] = x[r[at]].astype(np.float64) @ w[i].astype(np.float64).T
    z = sums * xs[r][:, None].astype(np.float64) * ws[e].astype(np.float64)
    want = z + (b[e].astype(np.float64) if bias else 0)
    # the sum's rounding, two products, the bias; below the range a step of it for each
    off = 3 * U * np.abs(z) + U * np.abs(want) + 4 * 2.0 ** -149
    if dtype == BF16:
        off = off + (np.abs(want) + off) * 2.0 ** -8 + 2.0 ** -133
    over = np.abs(want) - off > MOST
    unsure = ~over & (np.abs(want) + off > MOST * (1 - 2.0 ** -8))
    assert over.any() and (np.abs(got[over]) == np.inf).all() and (np.sign(got[over]) == np.sign(want[over])).all()
    ok = (np.abs(np.where(over | unsure, 0, got) - np.where(over | unsure, 0, want)) <= off)
    assert ok.all(), f"{int((~ok).sum())} of {ok.size}"


@gpu
@pytest.mark.parametrize("n,K", [(2, 3), (300, 3)])
def test_large_rows_and_small_weights(n, K):
    """Rows of 1e38 through weights of 1e-3, as quantize_rows gives both: the results of the fp32 product, up to the codes' rounding."""
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn(n, 64, generator=g).sign().cuda() * 1e38, torch.randn(K, 40, 64, generator=g).sign().cuda() * 1e-3
    ids = (torch.arange(n, dtype=torch.int32) % K).cuda()
    groups = pnn.group_rows(ids, K)
    got = pnn.grouped_forward_int8(groups, *pnn.quantize_rows(x), *pnn.quantize_rows(w))
    want = (w[ids.long()].double() @ x.double()[:, :, None])[:, :, 0]
    # (codes of 127 alone: the scales' roundings, the sum's and two products', of the terms' sizes at most)
    assert ((got.double() - want).abs() <= 6 * U * want.abs()).all()


@gpu
@pytest.mark.parametrize("n,k,K,I,O", SHAPES)
def test_powers_of_two_change_nothing_else(n, k, K, I, O):
    """A row's scale times 2^100 or 2^-100 is its results times that, to the bit, and its neighbours' results stay."""
    g = np.random.default_rng(n)
    x, w = (torch.from_numpy(g.integers(-127, 128, s).astype(np.int8)).cuda() for s in ((n, I), (K, O, I)))
    xs, ws = torch.from_numpy(scales((n,), [0, 1], 1)).cuda(), torch.from_numpy(scales((K, O), [-20, -19], 2)).cuda()
    b = torch.from_numpy(g.standard_normal((K, O)).astype(np.float32)).cuda()
    groups = pnn.group_rows(torch.from_numpy(g.integers(0, K, (n, k)).astype(np.int32)).cuda(), K)
    power = torch.from_numpy(g.choice([0, 0, 0, 100, -100], n)).cuda()
    plain = pnn.grouped_forward_int8(groups, x, xs, w, ws)
    got = pnn.grouped_forward_int8(groups, x, torch.ldexp(xs.double(), power).float(), w, ws)
    assert torch.equal(got, torch.ldexp(plain.double(), power.repeat_interleave(k)[:, None]).float())
    same = (power == 0).repeat_interleave(k)
    got = pnn.grouped_forward_int8(groups, x, torch.ldexp(xs.double(), power).float(), w, ws, b)
    assert torch.equal(got[same], pnn.grouped_forward_int8(groups, x, xs, w, ws, b)[same])
