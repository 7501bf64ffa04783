"""Results of pairs weighed into rows, and both gradients, against the formulas in 64 bits."""
import ctypes
import math

import pytest
import torch

from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
FAKE = 1 << 20


def args(**over):
    a = dict(y=FAKE, y_ld=10, type=pnn.FP32, width=10, n=4, per_row=2, networks=8, ids=FAKE, w=FAKE)
    a.update(over)
    return pnn.PnnCombine(*(a[f[0]] for f in pnn.PnnCombine._fields_))


BAD = [(dict(n=-1), pnn.PNN_ESHAPE), (dict(n=1 << 30), pnn.PNN_ESHAPE)] + [(d, pnn.PNN_EINVAL) for d in (
    dict(per_row=0), dict(networks=0), dict(networks=1025), dict(width=0), dict(width=(1 << 20) + 1), dict(y=None), dict(y=FAKE + 2),
    dict(y_ld=9), dict(type=2), dict(ids=None), dict(w=None), dict(ids=FAKE + 2), dict(w=FAKE + 1))]


@pytest.mark.parametrize("over,status", BAD)
def test_arguments_are_refused(over, status):
    L, a = pnn.lib(), args(**over)
    assert L.pnn_combine_rows(ctypes.byref(a), FAKE, 1 << 20, pnn.FP32, None) == status
    assert L.pnn_combine_grad(ctypes.byref(a), FAKE, 1 << 20, pnn.FP32, FAKE, 1 << 20, FAKE, None) == status
    assert L.pnn_last_error(None)


def test_memory_is_refused():
    L, a = pnn.lib(), args()
    assert L.pnn_combine_rows(None, FAKE, 10, pnn.FP32, None) == pnn.PNN_EINVAL
    for out, ld, kind in ((None, 10, 0), (FAKE + 2, 10, 0), (FAKE, 9, 0), (FAKE, 10, 3)):
        assert L.pnn_combine_rows(ctypes.byref(a), out, ld, kind, None) == pnn.PNN_EINVAL
    for g, ldg, dy, ldy, dw in ((None, 10, FAKE, 10, FAKE), (FAKE, 9, FAKE, 10, FAKE), (FAKE, 10, None, 10, FAKE),
                                (FAKE, 10, FAKE, 9, FAKE), (FAKE, 10, FAKE, 10, None), (FAKE, 10, FAKE, 10, FAKE + 2)):
        assert L.pnn_combine_grad(ctypes.byref(a), g, ldg, pnn.FP32, dy, ldy, dw, None) == pnn.PNN_EINVAL


def test_no_rows_need_no_device():
    a = args(n=0, y=None, ids=None, w=None)
    assert pnn.lib().pnn_combine_rows(ctypes.byref(a), None, 0, pnn.FP32, None) == pnn.PNN_OK
    assert pnn.lib().pnn_combine_grad(ctypes.byref(a), None, 0, pnn.FP32, None, 0, None, None) == pnn.PNN_OK


def test_the_binding_refuses():
    ids, w = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for y, i, g, why in ((torch.zeros(7, 3), ids, w, "y has shape"), (torch.zeros(8, 3), ids.long(), w, "ids is"),
                         (torch.zeros(8, 3), ids, w.double(), "gates is"), (torch.zeros(8, 3), ids, w[:, :1], "gates is"),
                         (torch.zeros(8), ids, w, "shapes"), (torch.zeros(8, 3), ids, w, "CUDA")):
        with pytest.raises(ValueError, match=why):
            pnn.combine_rows(y, i, g, 8)
        with pytest.raises(ValueError, match=why):
            pnn.combine_grad(torch.zeros(4, 3), y, i, g, 8)


def case(n, k, M, dtype, seed=0, pad=0, K=8):
    g = torch.Generator().manual_seed(seed)
    y = torch.randn(n * k, M + pad, generator=g).to(dtype).cuda()[:, pad:]
    dout = torch.randn(n, M + pad, generator=g).to(dtype).cuda()[:, pad:]
    ids = torch.randint(-1, K + 1, (n, k), generator=g, dtype=torch.int32)  # (-1 and K are outside)
    return y, dout, ids.cuda(), torch.randn(n, k, generator=g).cuda()


def near(got, want, off):
    if got.dtype == BF16:
        off = off + (want.abs() + off) * torch.finfo(BF16).eps / 2
    got = got.double().cpu()
    ok = (got - want).abs() <= off + 1e-37
    assert ok.all(), f"{int((~ok).sum())} of {ok.numel()}, largest {((got - want).abs() / off)[~ok].max():.3g} of the tolerance"


def verify(y, dout, ids, w, K=8, out_dtype=None):
    n, k = ids.shape
    M = y.shape[1]
    kept = ((ids >= 0) & (ids < K)).cpu()[:, :, None]
    y64 = torch.where(kept, y.double().cpu().view(n, k, M), 0.0)
    w64 = torch.where(kept, w.double().cpu()[:, :, None], 0.0)
    g64 = dout.double().cpu()[:, None, :]
    out = pnn.combine_rows(y, ids, w, K, out_dtype=out_dtype)
    assert out.dtype == (out_dtype or y.dtype)
    # a term passes through k fused additions
    near(out, (w64 * y64).sum(1), (w64 * y64).abs().sum(1) * (k + 1) * U)
    dy, dw = pnn.combine_grad(dout, y, ids, w, K)
    assert dy.dtype == y.dtype and dw.dtype == F32
    near(dy.view(n, k, M), torch.where(kept, w64 * g64, 0.0), (w64 * g64).abs() * U)
    # eight values a thread and step, then over the threads and waves
    near(dw, (y64 * g64).sum(2), (y64 * g64).abs().sum(2) * (8 * math.ceil(M / 2048) + 20) * U)
    assert (dy.view(n, k, M).cpu()[~kept.expand(n, k, M)] == 0).all() and (dw.cpu()[~kept[:, :, 0]] == 0).all()
    return out, dy, dw


SHAPES = [(1, 1, 1, 0), (5, 3, 2, 0), (33, 2, 7, 1), (40, 1, 64, 0), (17, 4, 203, 3), (9, 8, 511, 0), (7, 2, 512, 0), (3, 5, 1000, 5),
          (11, 2, 2048, 0), (4, 3, 4099, 1), (3000, 2, 40, 0), (2, 70, 33, 0), (9000, 2, 100, 0)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k,M,pad", SHAPES)
def test_rows_and_gradients(n, k, M, pad, dtype):
    y, dout, ids, w = case(n, k, M, dtype, pad=pad)
    verify(y, dout, ids, w)
    verify(y, dout.to(F32 if dtype == BF16 else BF16), ids, w, out_dtype=F32 if dtype == BF16 else BF16)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M", [7, 300, 3001])
def test_dropped_pairs_may_hold_anything(M, dtype):
    y, dout, ids, w = case(30, 3, M, dtype, seed=3)
    ids[4], ids[5], ids[6, 1] = -1, 2 ** 31 - 1, -2 ** 31
    dropped = (ids < 0) | (ids >= 8)
    y.view(30, 3, M)[dropped] = math.nan
    w[dropped] = math.inf
    out, dy, dw = verify(y, dout, ids, w)
    assert (out[4:6] == 0).all()
    dout[4] = math.nan  # (a row without a pair)
    dy, dw = pnn.combine_grad(dout, y, ids, w, 8)
    assert (dy.view(30, 3, M)[4] == 0).all() and (dw[4] == 0).all()
    y.view(30, 3, M)[9, 0] = math.inf  # a pair that is kept shows what it holds
    ids[9, 0] = 1
    assert not torch.isfinite(pnn.combine_rows(y, ids, w, 8)[9]).any()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M", [10, 700, 5000])
def test_in_place_and_strided(M, dtype):
    y, dout, ids, w = case(20, 2, M, dtype, seed=5, pad=1)
    want = pnn.combine_rows(y, ids, w, 8)
    dy, dw = pnn.combine_grad(dout, y, ids, w, 8)
    whole = torch.full((22, M + 7), 5.0, dtype=dtype, device="cuda")
    plain = whole.clone()
    pnn.combine_rows(y, ids, w, 8, out=whole[1:-1, 3:-4])
    plain[1:-1, 3:-4] = want
    assert torch.equal(whole, plain)
    got = pnn.combine_grad(dout, y, ids, w, 8, dy=y)
    assert got[0] is y and torch.equal(y, dy) and torch.equal(got[1], dw)


@gpu
def test_rows_behind_32_bits():
    n, k, M = 280_000, 2, 4096
    y = torch.ones(n * k, M, dtype=BF16, device="cuda")
    ids = torch.zeros(n, k, dtype=torch.int32, device="cuda")
    w = torch.full((n, k), 0.25, device="cuda")
    w[-1] = torch.tensor([2.0, -3.0])
    y[-1] = 4
    out = pnn.combine_rows(y, ids, w, 1)
    assert (out[:-1] == 0.5).all() and (out[-1] == -10).all()
    dy, dw = pnn.combine_grad(out, y, ids, w, 1, dy=y)
    assert (dw[:-1] == 2048).all() and dw[-1].tolist() == [-40960.0, -163840.0]
    assert (dy[-2] == -20).all() and (dy[-1] == 30).all() and (dy[:-2] == 0.125).all()


@gpu
def test_another_stream_a_graph_and_the_same_bits():
    y, dout, ids, w = case(3000, 3, 1000, BF16)

    def step(stream=None):
        return (pnn.combine_rows(y, ids, w, 8, stream=stream), *pnn.combine_grad(dout, y, ids, w, 8, stream=stream))

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for _ in range(4):
        y.mul_(-0.75)
        w.add_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(kept, step()):
            assert torch.equal(a, b)
