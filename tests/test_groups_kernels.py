"""Every kernel that a rule on sizes selects for the grouped products, at contractions that go round its ring of
stages several times, ragged in all three extents, with every activation's slope; unequal groups."""
import pytest
import torch

from paper_2304_09590_amd import pnn
from tests.test_groups import ACTS, BF16, F32, Case, close, slope

gpu = pytest.mark.gpu

# n, per_row, networks, inputs, outputs, pad (odd pads: rows off 16 bytes)
SHAPES = [
    (9000, 1, 5, 520, 1736, 0), (9000, 1, 5, 1736, 520, 0), (9000, 1, 5, 519, 1735, 1), (9000, 1, 5, 1735, 519, 1),
    (4500, 1, 5, 1736, 1800, 0), (4500, 2, 9, 1096, 1032, 0), (12000, 1, 32, 1000, 1096, 0), (12000, 1, 32, 1096, 1000, 0), (6000, 2, 32, 1096, 1000, 0),
    (12000, 1, 32, 999, 1095, 3), (3000, 1, 3, 264, 136, 0), (2000, 2, 5, 136, 328, 8), (700, 1, 9, 328, 72, 0)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,per_row,networks,inputs,outputs,pad", SHAPES)
def test_products(n, per_row, networks, inputs, outputs, pad, dtype):
    c = Case(n, per_row, networks, inputs, outputs, dtype, pad=pad, seed=37)
    for act, out_dtype in ((pnn.RELU, None), (pnn.TANH, F32), (None, BF16)):
        want, size = c.forward(act, 1.0)
        got = pnn.grouped_forward(c.groups, c.x, c.w, c.b, act=act, out_dtype=out_dtype)
        close(got, want, size, inputs, act)
        assert (got[~c.kept] == 0).all()
    want, size = c.backward_input()
    for act, out_dtype in ((None, F32), (pnn.SIGMOID, None), (pnn.TANH, F32), (pnn.RELU, None), (pnn.LEAKY_RELU, BF16)):
        a = s = None
        if act is not None:
            a = ACTS[act](c.x.double())
            a = (torch.where(c.x < 0, -a.abs(), a) if act in (pnn.RELU, pnn.LEAKY_RELU) else a).to(dtype)
            s = slope(act, a.double())
        got = pnn.grouped_backward_input(c.groups, c.dy, c.w, a=a, act=act, out_dtype=out_dtype)
        close(got, want * s if act is not None else want, size * (s.abs() + 2.0 ** -23) if act is not None else size,
              outputs * per_row + 64)
    dw, db = pnn.grouped_backward_weights(c.groups, c.dy, c.x)
    want, size, bwant, bsize = c.backward_weights()
    close(dw, want, size, n * per_row)
    close(db, bwant, bsize, n * per_row)


def skewed(n, networks, popular, seed=41):
    """Most rows name one network, the others share the rest; some none."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, networks, (n, 1), generator=g, dtype=torch.int32)
    ids[torch.rand(n, 1, generator=g) < 0.8] = popular
    ids[torch.rand(n, 1, generator=g) < 0.05] = -1
    return ids


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,networks,inputs,outputs,pad", [
    (100, 64, 104, 72, 0), (100, 64, 103, 71, 1), (2000, 256, 136, 72, 0), (9000, 33, 264, 328, 0), (9000, 33, 263, 327, 1), (5000, 3, 520, 1032, 0)])
def test_unequal_groups(n, networks, inputs, outputs, pad, dtype):
    """One network holds most pairs: many tiles of 16 of it, one long group among short ones."""
    c = Case(n, 1, networks, inputs, outputs, dtype, pad=pad, seed=43)
    c.ids = skewed(n, networks, networks - 2)
    c.groups = pnn.group_rows(c.ids.cuda(), networks)
    flat = c.ids.reshape(-1)
    c.kept = ((flat >= 0) & (flat < networks)).cuda()
    c.members = [torch.nonzero(flat == e)[:, 0].cuda() for e in range(networks)]
    want, size = c.forward(pnn.SIGMOID, 1.0)
    got = pnn.grouped_forward(c.groups, c.x, c.w, c.b, act=pnn.SIGMOID)
    close(got, want, size, inputs, pnn.SIGMOID)
    assert (got[~c.kept] == 0).all()
    want, size = c.backward_input()
    a = torch.tanh(c.x.double()).to(dtype)
    s = slope(pnn.TANH, a.double())
    close(pnn.grouped_backward_input(c.groups, c.dy, c.w, a=a, act=pnn.TANH), want * s, size * (s.abs() + 2.0 ** -23), outputs + 64)
    dw, db = pnn.grouped_backward_weights(c.groups, c.dy, c.x)
    want, size, bwant, bsize = c.backward_weights()
    close(dw, want, size, n)
    close(db, bwant, bsize, n)


def names_of(call):
    """Device kernels that a call runs, as the profiler names them."""
    from torch.profiler import ProfilerActivity, profile
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    return [e.name for e in p.events() if "group_" in e.name]


RING = {"256x256": "256, 256, 2, 4", "256x128": "256, 128, 2, 2", "128x64": "128, 64, 2, 2"}


# sizes as above and the kernels of the three directions
@gpu
@pytest.mark.parametrize("dtype,shape,kernels", [
    (BF16, (9000, 1, 5, 520, 1736, 0), ("ring 256x256", "ring 128x64", "ring 256x256")),
    (BF16, (9000, 1, 5, 1736, 520, 0), ("ring 128x64", "ring 256x256", "ring 256x256")),
    (BF16, (12000, 1, 32, 1000, 1096, 0), ("ring 256x128", "ring 128x64", "ring 256x128")),
    (BF16, (12000, 1, 32, 1096, 1000, 0), ("ring 128x64", "ring 256x128", "ring 256x128")),
    (BF16, (3000, 1, 3, 264, 136, 0), ("ring 128x64", "ring 128x64", "ring 128x64")),
    (BF16, (12000, 1, 32, 999, 1095, 3), ("tile 128", "tile 128", "tile 128")),
    (F32, (12000, 1, 32, 1000, 1096, 0), ("tile 128", "tile 128", "tile 128")),
    (F32, (700, 1, 9, 328, 72, 0), ("tile 64", "tile 64", "tile 64")),
    (F32, (100, 1, 64, 104, 72, 0), ("few", "few", "tile 64")),
    (BF16, (100, 1, 64, 104, 72, 0), ("few", "few", "ring 128x64"))])
def test_the_kernels_that_run(dtype, shape, kernels):
    c = Case(*shape[:5], dtype, pad=shape[5], seed=47)
    calls = (lambda: pnn.grouped_forward(c.groups, c.x, c.w, c.b), lambda: pnn.grouped_backward_input(c.groups, c.dy, c.w),
             lambda: pnn.grouped_backward_weights(c.groups, c.dy, c.x))
    for direction, (call, kernel) in enumerate(zip(calls, kernels)):
        kind, _, size = kernel.partition(" ")
        names = names_of(call)
        if kind == "few":
            want = ("group_few_fwd_kernel<", "group_few_dx_kernel<")[direction]
        elif kind == "ring":
            want = f"{direction}, "
            names = [n for n in names if "group_ring_kernel<" in n and f", {RING[size]}, " in n]
        else:
            want = f"{direction}, "
            names = [n for n in names if "group_tile_kernel<" in n and f", {size}>" in n]
        assert any(want in n for n in names), (direction, kernel, names_of(call))
