"""Rows as 8-bit codes, and the grouped product of codes, against the formulas in 64 bits."""
import ctypes
import math

import pytest
import torch

from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
FAKE = 1 << 20


# ---- refusals, on the host -----------------------------------------------------------------------

def test_rows_are_refused():
    L = pnn.lib()
    good = dict(x=FAKE, x_ld=20, type=pnn.FP32, n=4, width=20, q=FAKE, q_ld=32, scale=FAKE)
    for over, status in ((dict(n=-1), pnn.PNN_ESHAPE), (dict(width=0), pnn.PNN_EINVAL), (dict(width=(1 << 20) + 1), pnn.PNN_EINVAL),
                         (dict(x=None), pnn.PNN_EINVAL), (dict(x=FAKE + 2), pnn.PNN_EINVAL), (dict(x_ld=19), pnn.PNN_EINVAL),
                         (dict(type=2), pnn.PNN_EINVAL), (dict(q=None), pnn.PNN_EINVAL), (dict(q=FAKE + 8), pnn.PNN_EINVAL),
                         (dict(q_ld=40), pnn.PNN_EINVAL), (dict(q_ld=16), pnn.PNN_EINVAL), (dict(scale=None), pnn.PNN_EINVAL),
                         (dict(scale=FAKE + 1), pnn.PNN_EINVAL), (dict(n=0, x=None, q=None, scale=None), pnn.PNN_OK)):
        assert L.pnn_quantize_rows(*{**good, **over}.values(), None) == status, over


GROUPS = dict(plan=FAKE, n=4, per_row=2, networks=3)
LAYER = dict(inputs=32, outputs=5, w=FAKE, w_net=160, w_ld=32, scale=FAKE, scale_net=5, b=FAKE, b_net=5)
CALL = dict(x=FAKE, x_ld=32, x_scale=FAKE, act=-1, y=FAKE, y_ld=5, y_type=pnn.FP32)
BAD = [("groups", dict(n=-1), pnn.PNN_ESHAPE)] + [(w, d, pnn.PNN_EINVAL) for w, d in (
    ("groups", dict(networks=0)), ("groups", dict(per_row=0)), ("groups", dict(plan=None)), ("layer", dict(inputs=0)),
    ("layer", dict(inputs=24)), ("layer", dict(inputs=(1 << 17) + 16, w_ld=1 << 18)), ("layer", dict(outputs=0)),
    ("layer", dict(outputs=(1 << 20) + 1)), ("layer", dict(w=None)), ("layer", dict(w=FAKE + 8)), ("layer", dict(w_ld=16)),
    ("layer", dict(w_ld=40)), ("layer", dict(w_net=-16)), ("layer", dict(w_net=168)), ("layer", dict(scale=None)),
    ("layer", dict(scale=FAKE + 2)), ("layer", dict(scale_net=-1)), ("layer", dict(b=FAKE + 2)), ("layer", dict(b_net=-1)),
    ("call", dict(act=pnn.SOFTMAX)), ("call", dict(act=-2)), ("call", dict(x=None)), ("call", dict(x=FAKE + 4)), ("call", dict(x_ld=31)),
    ("call", dict(x_ld=40)), ("call", dict(x_scale=None)), ("call", dict(x_scale=FAKE + 2)), ("call", dict(y=None)),
    ("call", dict(y=FAKE + 2)), ("call", dict(y_ld=4)), ("call", dict(y_type=2)))]


@pytest.mark.parametrize("which,over,status", BAD)
def test_products_are_refused(which, over, status):
    a = {"groups": GROUPS, "layer": LAYER, "call": CALL}
    a[which] = {**a[which], **over}
    g, w = pnn.PnnGroups(*a["groups"].values()), pnn.PnnGroupCodes(*a["layer"].values())
    assert pnn.lib().pnn_grouped_forward_int8(ctypes.byref(g), ctypes.byref(w), *a["call"].values(), None) == status
    assert pnn.lib().pnn_last_error(None)
    assert pnn.lib().pnn_grouped_forward_int8(None, ctypes.byref(w), *a["call"].values(), None) == pnn.PNN_EINVAL
    assert pnn.lib().pnn_grouped_forward_int8(ctypes.byref(pnn.PnnGroups(*GROUPS.values())), None, *a["call"].values(), None) == pnn.PNN_EINVAL


def test_no_rows_need_no_device():
    g, w = pnn.PnnGroups(None, 0, 2, 3), pnn.PnnGroupCodes(*LAYER.values())
    assert pnn.lib().pnn_grouped_forward_int8(ctypes.byref(g), ctypes.byref(w), None, 0, None, -1, None, 0, 0, None) == pnn.PNN_OK


def test_the_binding_refuses():
    for x, why in ((torch.zeros(4), "expected rows"), (torch.zeros(4, 0), "expected rows"), (torch.zeros(8, 4).T, "not contiguous"),
                   (torch.zeros(3, 4, 8)[:, :, :4], "stack"), (torch.zeros(4, 8, dtype=torch.float64), "float32 or bfloat16"),
                   (torch.zeros(4, 8), "CUDA")):
        with pytest.raises(ValueError, match=why):
            pnn.quantize_rows(x)
    groups = pnn.RowGroups(torch.zeros(64, dtype=torch.int32), 4, 1, 2)
    x, xs, w, ws = torch.zeros(4, 16, dtype=torch.int8), torch.zeros(4), torch.zeros(2, 5, 16, dtype=torch.int8), torch.zeros(2, 5)
    for a, why in (((x, xs, w[0], ws), "w has shape"), ((x, xs, w.float(), ws), "w is"), ((x, xs, w, ws[:, :4]), "w_scale has"),
                   ((x, xs, w, ws.double()), "w_scale is"), ((x, xs, w, ws, ws[:1]), "b has shape"), ((x, xs, w, ws), "CUDA")):
        with pytest.raises(ValueError, match=why):
            pnn.grouped_forward_int8(groups, *a)


# ---- codes ---------------------------------------------------------------------------------------

def codes_of(x):
    """Codes and scales in 64 bits."""
    x = x.double().cpu()
    top = x.abs().amax(-1, keepdim=True)
    # (127 x is exact in 64 bits and a quotient in the middle between two integers is, too: ties are ties)
    q = torch.where(top > 0, torch.round(127 * x / torch.where(top > 0, top, 1.0)), 0.0)
    return torch.nn.functional.pad(q, (0, -x.shape[-1] % 16)).to(torch.int8), (top[..., 0].float() / 127)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape,pad", [((1, 1), 0), ((3, 16), 0), ((5, 17), 1), ((33, 255), 0), ((9, 257), 3), ((40, 784), 0), ((7, 1025), 0),
                                       ((4, 4096), 0), ((4, 4097), 1), ((2, 20000), 0), ((9000, 33), 0), ((3, 5, 70), 0), ((9000, 2000), 0)])
def test_codes(shape, pad, dtype):
    g = torch.Generator().manual_seed(1)
    x = torch.randn(*shape[:-1], shape[-1] + pad, generator=g) * torch.exp(3 * torch.randn(*shape[:-1], 1, generator=g))
    x = x.to(dtype).cuda()[..., pad:]
    q, s = pnn.quantize_rows(x)
    want, scale = codes_of(x)
    assert torch.equal(q.cpu(), want) and torch.equal(s.cpu(), scale)


@gpu
@pytest.mark.parametrize("width", [5, 300, 1030, 2000, 4000, 5000])
def test_codes_of_extremes(width):
    x = torch.randn(20, width, generator=torch.Generator().manual_seed(2))
    x[0] = 0
    x[1] = -0.0
    x[2], x[2, 3] = 0, 1e-45
    x[3] *= 1e-41
    x[4] *= 1e37
    x[5, 0] = torch.finfo(F32).max
    x[6] = 127.0 / 2
    x[6, 0], x[6, 1], x[6, 2] = 127.0, 0.5, -1.5  # in the middle between two: to the even one
    x = x.cuda()
    q, s = pnn.quantize_rows(x)
    want, scale = codes_of(x)
    assert torch.equal(q.cpu(), want) and torch.equal(s.cpu(), scale) and q[6, :3].tolist() == [127, 0, -2]
    x[7, width - 1], x[8, 0], x[9, 2] = math.nan, math.inf, -math.inf
    q, s = pnn.quantize_rows(x)
    assert (q[7:10] == 0).all() and torch.isnan(s[7:10]).all() and torch.equal(q[10:].cpu(), want[10:]) and torch.isfinite(s[10:]).all()


# ---- products ------------------------------------------------------------------------------------

ACTS = {"none": None, "sigmoid": pnn.SIGMOID, "tanh": pnn.TANH, "relu": pnn.RELU, "leaky": pnn.LEAKY_RELU}


def value_of(name, z):
    return {"none": lambda v: v, "sigmoid": torch.sigmoid, "tanh": torch.tanh, "relu": lambda v: v.clamp(min=0),
            "leaky": lambda v: torch.where(v < 0, 0.01 * v, v)}[name](z)


def case(n, k, K, I, O, seed=0, even=False):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0 if even else -1, K if even else K + 1, (n, k), generator=g, dtype=torch.int32)  # (-1 and K are dropped)
    x = torch.randint(-127, 128, (n, I), generator=g, dtype=torch.int8)
    w = torch.randint(-127, 128, (K, O, I), generator=g, dtype=torch.int8)
    xs, ws = torch.rand(n, generator=g) * 0.02, torch.rand(K, O, generator=g) * 0.02 / math.sqrt(I)
    return [t.cuda() for t in (ids, x, xs, w, ws, torch.randn(K, O, generator=g))]


def verify(ids, x, xs, w, ws, b, act, dtype, K, out=None):
    n, k = ids.shape
    groups = pnn.group_rows(ids, K)
    y = pnn.grouped_forward_int8(groups, x, xs, w, ws, b, act=ACTS[act], out_dtype=None if out is not None else dtype, out=out)
    assert y.dtype == dtype
    flat = ids.flatten().cpu().long()
    kept = (flat >= 0) & (flat < K)
    rows = torch.arange(n * k) // k
    want, off = (torch.zeros(n * k, w.shape[1], dtype=torch.float64) for _ in range(2))
    for e in range(K):
        at = torch.nonzero(flat == e)[:, 0]
        if at.numel() == 0:
            continue
        sums = (x[rows[at].cuda()].double() @ w[e].double().T).cpu()
        z = sums * xs.double().cpu()[rows[at]][:, None] * ws[e].double().cpu()
        # the sum's rounding, two products, the bias
        o = 3 * U * z.abs()
        if b is not None:
            z = z + b[e].double().cpu()
        want[at] = value_of(act, z)
        off[at] = o + U * z.abs() + (0 if act in ("none", "relu") else 6 * U * (1 + want[at].abs()))
    if dtype == BF16:
        off = off + (want.abs() + off) * torch.finfo(BF16).eps / 2
    ok = (y.double().cpu() - want).abs() <= off + 1e-37
    assert ok.all(), f"{int((~ok).sum())} of {ok.numel()} at {torch.nonzero(~ok)[:3].tolist()}"
    assert (y.cpu()[~kept] == 0).all()
    return groups, y


# (pairs a network in the mean: at most two, tiles of 128 x 64, 256 x 128, 256 x 256)
SHAPES = [(1, 1, 1, 16, 1), (1, 2, 64, 784, 512), (5, 2, 9, 48, 33), (3, 3, 40, 2064, 70), (33, 1, 3, 16, 17), (70, 2, 5, 80, 203), (129, 1, 2, 512, 64),
          (400, 3, 7, 1008, 130), (4096, 1, 16, 96, 3329), (2500, 2, 20, 208, 2600), (8192, 1, 2, 64, 2049), (5000, 2, 4, 176, 1031), (1200, 1, 1, 1040, 24000)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k,K,I,O", SHAPES)
def test_products(n, k, K, I, O, dtype):
    ids, x, xs, w, ws, b = case(n, k, K, I, O)
    for act, bias in (("relu", b), ("none", None)):
        verify(ids, x, xs, w, ws, bias, act, dtype, K)


@gpu
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("n,k,K,I,O", [(5, 2, 9, 48, 33), (70, 2, 5, 80, 203), (4096, 1, 16, 96, 3329), (8192, 1, 2, 64, 2049)])
def test_activations(n, k, K, I, O, act):
    ids, x, xs, w, ws, b = case(n, k, K, I, O, seed=2)
    verify(ids, x, xs, w, ws, b, act, F32, K)


@gpu
@pytest.mark.parametrize("n,K,I", [(2, 3, 1 << 17), (40, 2, 1 << 17)])
def test_the_largest_sums(n, K, I):
    """127 x 127 x 2^17 is below 2^31: no sum overflows."""
    ids = (torch.arange(n, dtype=torch.int32) % K).view(n, 1).cuda()
    x = torch.full((n, I), 127, dtype=torch.int8, device="cuda")
    w = torch.full((K, 20, I), 127, dtype=torch.int8, device="cuda")
    w[0] = -127
    one = torch.ones(n, device="cuda")
    y = pnn.grouped_forward_int8(pnn.group_rows(ids, K), x, one, w, torch.ones(K, 20, device="cuda"))
    want = torch.where(ids == 0, -1.0, 1.0) * float(127 * 127 * I)
    assert (y == want).all()


@gpu
@pytest.mark.parametrize("n,k,K,I,O", [(3, 2, 9, 48, 33), (70, 2, 5, 80, 203), (4096, 1, 16, 96, 3329), (8192, 1, 2, 64, 2049)])
def test_strides_and_rows_of_dropped_pairs(n, k, K, I, O):
    """Rows, networks and results further apart than they are wide; scales of NaN show, dropped pairs do not."""
    ids, x, xs, w, ws, b = case(n, k, K, I, O, seed=4)
    xw = torch.full((n, I + 32), 99, dtype=torch.int8, device="cuda")
    xw[:, 16:-16] = x
    ww = torch.full((K, O + 1, I + 16), 77, dtype=torch.int8, device="cuda")
    ww[:, :-1, :-16] = w
    sw = torch.full((K, O + 3), math.nan, device="cuda")
    sw[:, 1:-2] = ws
    whole = torch.full((n * k + 2, O + 5), 5.0, device="cuda")
    _, y = verify(ids, xw[:, 16:-16], xs, ww[:, :-1, :-16], sw[:, 1:-2], b, "relu", F32, K, out=whole[1:-1, 2:-3])
    plain = torch.full_like(whole, 5.0)
    plain[1:-1, 2:-3] = y
    assert torch.equal(whole, plain)
    ids[1] = -1
    ids[2] = 0
    xs[1], xs[2] = math.nan, math.nan
    y = pnn.grouped_forward_int8(pnn.group_rows(ids, K), x, xs, w, ws, b).view(n, k, O)
    assert (y[1] == 0).all() and torch.isnan(y[2]).all() and torch.isfinite(y[3:]).all()


@gpu
def test_one_set_of_weights_for_all_networks():
    ids, x, xs, w, ws, b = case(40, 2, 6, 64, 50, seed=6)
    w, ws, b = (t[:1].expand(6, *t.shape[1:]) for t in (w, ws, b))
    verify(ids, x, xs, w, ws, b, "none", F32, 6)


@gpu
def test_results_behind_32_bits():
    n, K, I, O = 70000, 4, 16, 32768
    ids, x, xs, w, ws, b = case(n, 1, K, I, O, seed=8)
    y = pnn.grouped_forward_int8(pnn.group_rows(ids, K), x, xs, w, ws, b, out_dtype=BF16)
    at = torch.tensor([0, 1, 65535, 65536, n - 2, n - 1], device="cuda")
    z = torch.stack([(x[r].double() @ w[int(ids[r])].double().T) * xs[r].double() * ws[int(ids[r])].double() + b[int(ids[r])].double()
                     if 0 <= int(ids[r]) < K else torch.zeros(O, dtype=torch.float64, device="cuda") for r in at.tolist()])
    assert ((y[at].double() - z).abs() <= z.abs() * (2.0 ** -8 + 4 * U) + 4 * U * 4).all()


@gpu
@pytest.mark.parametrize("dtype,n", [(BF16, 25000), (F32, 35000)])
def test_results_larger_than_the_caches(dtype, n):
    """An odd number of outputs and a distance between rows that is no multiple of 16 bytes; what lies beside stays."""
    K, I, O = 5, 64, 2047
    ids, x, xs, w, ws, b = case(n, 1, K, I, O, seed=10)
    whole = torch.full((n, O + 2), 5.0, dtype=dtype, device="cuda")
    assert n * O * whole.element_size() > (96 if dtype == BF16 else 256) << 20
    verify(ids, x, xs, w, ws, b, "relu", dtype, K, out=whole[:, 1:-1])
    assert (whole[:, 0] == 5).all() and (whole[:, -1] == 5).all()


@gpu
def test_rows_to_answers_on_another_stream_and_in_a_graph():
    """Two layers as a program serves them: codes of the rows, the product, codes of its results, the next product."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(300, 100, generator=g, device="cuda")
    w1, w2 = torch.randn(7, 60, 100, generator=g, device="cuda"), torch.randn(7, 10, 60, generator=g, device="cuda")
    b1 = torch.randn(7, 60, generator=g, device="cuda")
    ids = torch.randint(0, 7, (300, 2), generator=g, device="cuda", dtype=torch.int32)
    c1, c2 = pnn.quantize_rows(w1), pnn.quantize_rows(w2)

    def step(stream=None):
        groups = pnn.group_rows(ids, 7, stream=stream)
        pairs = pnn.RowGroups(groups.plan, 600, 1, 7, groups.stream)
        q = pnn.quantize_rows(x, stream=stream)
        h = pnn.grouped_forward_int8(groups, *q, *c1, b1, act=pnn.RELU, out_dtype=BF16, stream=stream)
        return h, pnn.grouped_forward_int8(pairs, *pnn.quantize_rows(h, stream=stream), *c2, stream=stream)

    want = step()
    # (off by the codes' roundings: half a code of both operands)
    e = ids.flatten().long()
    z = torch.relu((w1[e].double() @ x.repeat_interleave(2, 0).double()[:, :, None])[:, :, 0] + b1[e].double())
    assert (want[0].double() - z).norm() <= 0.02 * z.norm()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for _ in range(4):
        x.mul_(-0.75)
        ids.copy_((ids + 1) % 7)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(kept, step()):
            assert torch.equal(a, b)
