"""The distillation loss from a teacher's top logits and its gradient, against the formulas in 64 bits
and against differences."""
import ctypes
import math

import pytest
import torch

from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24  # half a step of fp32
FAKE = 1 << 20


# ---- refusals, on the host -----------------------------------------------------------------------

def args(**over):
    a = dict(z=FAKE, z_ld=10, type=pnn.FP32, classes=10, n=4, idx=FAKE, t=FAKE, top=3, y=None, temperature=2.0, alpha=0.0)
    a.update(over)
    return pnn.PnnDistill(*(a[f[0]] for f in pnn.PnnDistill._fields_))


BAD = [(dict(n=-1), pnn.PNN_ESHAPE), (dict(n=1 << 31), pnn.PNN_ESHAPE)] + [(d, pnn.PNN_EINVAL) for d in (
    dict(classes=0), dict(classes=(1 << 30) + 1), dict(top=-1), dict(top=1025), dict(temperature=0.0), dict(temperature=-1.0),
    dict(temperature=math.nan), dict(temperature=math.inf), dict(alpha=-0.1), dict(alpha=1.5), dict(alpha=math.nan),
    dict(z=None), dict(z=FAKE + 2), dict(z_ld=9), dict(type=2), dict(idx=None), dict(t=None), dict(idx=FAKE + 2),
    dict(t=FAKE + 2), dict(alpha=0.5), dict(alpha=0.5, y=FAKE + 1))]


@pytest.mark.parametrize("over,status", BAD)
def test_arguments_are_refused(over, status):
    L, a = pnn.lib(), args(**over)
    assert L.pnn_distill_loss(ctypes.byref(a), FAKE, FAKE, 1 << 40, None) == status
    assert L.pnn_distill_grad(ctypes.byref(a), None, FAKE, 1 << 40, FAKE, 10, None) == status
    assert L.pnn_last_error(None)


def test_memory_is_refused():
    L, a, size = pnn.lib(), args(), ctypes.c_int64()
    assert L.pnn_distill_bytes(4, 10, ctypes.byref(size)) == pnn.PNN_OK and size.value == 64
    assert L.pnn_distill_bytes(4, 10, None) == pnn.PNN_EINVAL
    assert L.pnn_distill_bytes(4, 0, ctypes.byref(size)) == pnn.PNN_EINVAL
    assert L.pnn_distill_loss(None, FAKE, FAKE, 64, None) == pnn.PNN_EINVAL
    for loss, stats, have, status in ((None, FAKE, 64, pnn.PNN_EINVAL), (FAKE + 2, FAKE, 64, pnn.PNN_EINVAL),
                                      (FAKE, None, 64, pnn.PNN_EINVAL), (FAKE, FAKE + 8, 64, pnn.PNN_EINVAL),
                                      (FAKE, FAKE, 63, pnn.PNN_ESHAPE)):
        assert L.pnn_distill_loss(ctypes.byref(a), loss, stats, have, None) == status
    for g, dz, ld in ((FAKE + 2, FAKE, 10), (None, None, 10), (None, FAKE + 2, 10), (None, FAKE, 9)):
        assert L.pnn_distill_grad(ctypes.byref(a), g, FAKE, 64, dz, ld, None) == pnn.PNN_EINVAL


def test_no_rows_need_no_device():
    a = args(n=0, z=None, idx=None, t=None)
    assert pnn.lib().pnn_distill_loss(ctypes.byref(a), None, None, 0, None) == pnn.PNN_OK
    assert pnn.lib().pnn_distill_grad(ctypes.byref(a), None, None, 0, None, 0, None) == pnn.PNN_OK


# ---- values --------------------------------------------------------------------------------------

def reference(z, idx, t, y, temperature, alpha, g):
    """Loss, gradient and what each may be off by.  An exponential of d is off by a step or two and 2 |d| U (the
    difference, its scaling); a sum by its terms' errors and a step for each of the additions that a value passes
    through; a logarithm by its argument's relative error and a step of its own."""
    n, v = z.shape
    z, t, g = z.double().cpu(), t.double().cpu(), g.double().cpu()
    idx = idx.long().cpu()
    adds = math.ceil(v / 512) * 8 + 40
    kept = (idx >= 0) & (idx < v)
    at = torch.where(kept, idx, 0)

    def softmax(x, scale):
        d = (x - x.max(1, keepdim=True).values) * scale
        e = torch.exp(d)
        q = e / e.sum(1, keepdim=True)
        size = torch.where(q > 0, d.abs(), torch.zeros_like(d))  # (-inf has no weight)
        off = ((2 * (q * size).sum(1, keepdim=True)) + adds) * U  # of the sum, relative
        return d - torch.log(e.sum(1, keepdim=True)), q, size, off

    lq, q, dq, offq = softmax(z, 1 / temperature)
    masked = torch.where(kept, t, torch.full_like(t, -math.inf))
    loss, tol = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    dz, dtol = torch.zeros_like(z), torch.zeros_like(z)
    dead = torch.isinf(z).all(1)
    if idx.shape[1] and alpha < 1:
        some = torch.isfinite(masked).any(1) & ~dead
        lp, p, dp, offp = softmax(masked, 1 / temperature)
        zero = torch.zeros_like(p)
        live = kept & (p > 0)
        gap = torch.where(live, lp - lq.gather(1, at), zero)
        p = torch.where(live, p, zero)
        size = torch.where(live, lp.abs() + lq.gather(1, at).abs(), zero)
        w = (1 - alpha) * temperature ** 2
        kl = (p * gap).sum(1)
        koff = (p * (gap.abs() * (2 * dp + offp / U + 8) * U + (8 * size + 8) * U + offp + offq)).sum(1) + (p * gap.abs()).sum(1) * 20 * U
        loss += torch.where(some, w * kl, 0.0)
        tol += torch.where(some, w * koff, 0.0)
        mass = torch.zeros_like(z).scatter_add(1, at, p)
        moff = torch.zeros_like(z).scatter_add(1, at, p * ((2 * dp + 30) * U + offp))
        part = (1 - alpha) * temperature * (q - mass)
        poff = (1 - alpha) * temperature * (q * ((2 * dq + 8) * U + offq) + moff + 4 * U * (q + mass))
        dz += torch.where(some[:, None], part, 0.0)
        dtol += torch.where(some[:, None], poff, 0.0)
    if y is not None and alpha > 0:
        y = y.long().cpu()
        some = (y >= 0) & (y < v) & ~dead
        yc = torch.where(some, y, 0)[:, None]
        ls, s, ds, offs = softmax(z, 1.0)
        lab = ls.gather(1, yc)
        loss += torch.where(some, -alpha * lab[:, 0], 0.0)
        tol += torch.where(some, alpha * ((8 * lab.abs() + 8) * U + offs)[:, 0], 0.0)
        hot = torch.zeros_like(z).scatter(1, yc, 1.0)
        dz += torch.where(some[:, None], alpha * (s - hot), 0.0)
        dtol += torch.where(some[:, None], alpha * (s * ((2 * ds + 8) * U + offs) + 4 * U * (s + hot)), 0.0)
    tol = tol + 4 * U * loss.abs() + 1e-37
    return loss, tol, dz * g[:, None], (dtol + 4 * U * dz.abs()) * g.abs()[:, None] + 1e-37


def case(n, v, k, dtype, seed=0, pad=0, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn(n, v + pad, generator=g) * scale).to(dtype).cuda()[:, pad:]
    idx = torch.stack([torch.randperm(v, generator=g)[:k] if k <= v else torch.randint(0, v, (k,), generator=g)
                       for _ in range(n)]).to(torch.int32).reshape(n, k)
    t = (torch.randn(n, k, generator=g) * scale).to(dtype)
    y = torch.randint(0, v, (n,), generator=g, dtype=torch.int32)
    grad = torch.randn(n, generator=g)
    return z, idx.cuda(), t.cuda(), y.cuda(), grad.cuda()


def verify(z, idx, t, y, g, temperature, alpha):
    loss, stats = pnn.distill_loss(z, idx, t, y=y, temperature=temperature, alpha=alpha)
    dz = pnn.distill_grad(z, idx, t, stats, g, y=y, temperature=temperature, alpha=alpha)
    want, tol, dwant, dtol = reference(z, idx, t, y, temperature, alpha, g)
    assert dz.dtype == z.dtype and loss.dtype == F32
    if z.dtype == BF16:
        dtol = dtol + (dwant.abs() + dtol) * torch.finfo(BF16).eps / 2
    for got, value, off in ((loss, want, tol), (dz, dwant, dtol)):
        got = got.double().cpu()
        ok = ((got - value).abs() <= off) | (got == value)
        assert ok.all(), f"{int((~ok).sum())} of {ok.numel()}, largest {((got - value).abs() / off)[~ok].max():.3g} of the tolerance"
    return loss, dz


SHAPES = [(1, 1, 1, 0), (3, 2, 2, 0), (60, 10, 3, 0), (17, 16, 16, 1), (33, 17, 5, 0), (20, 128, 16, 3), (20, 129, 7, 0),
          (20, 100, 17, 0), (9, 1000, 64, 0), (9, 1001, 65, 1), (3, 50, 200, 0), (5, 2048, 8, 0), (5, 2049, 8, 3), (2, 4104, 1024, 0),
          (1, 131071, 20, 0), (7, 20000, 33, 5), (1100, 4100, 4, 0)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,k,pad", SHAPES)
def test_loss_and_gradient(n, v, k, pad, dtype):
    z, idx, t, y, g = case(n, v, k, dtype, pad=pad)
    for temperature, alpha in ((2.0, 0.25), (1.0, 0.5), (0.5, 0.0), (3.0, 1.0)):
        verify(z, idx, t, y if alpha > 0 else None, g, temperature, alpha)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,k", [(40, 12, 6), (40, 700, 40), (12, 9000, 90)])
def test_padding_repeated_classes_and_rows_without_entries(n, v, k, dtype):
    z, idx, t, y, g = case(n, v, k, dtype, seed=5)
    idx[:, 1] = idx[:, 0]                      # a class that stands twice
    idx[2, :] = idx[2, 0]                      # one class in all entries
    idx[3:20, k // 2:] = -1                    # padding, and what it may hold
    idx[4, k // 2:] = v
    idx[5, k // 2:] = -2 ** 31
    t[3:20, k // 2:] = math.nan
    idx[6] = -1                                # no entries
    y[7], y[8], y[9] = -1, v, 2 ** 31 - 1      # no label
    idx[9] = -1                                # neither
    t[10, 0] = -math.inf                       # an entry without weight
    t[11] = -math.inf                          # none with weight
    y[0] = idx[0, 0]                           # the label is an entry's class
    g[1] = 0
    for temperature, alpha in ((2.0, 0.25), (1.5, 0.0)):
        loss, dz = verify(z, idx, t, y, g, temperature, alpha)
        assert loss[9] == 0 and (dz[9] == 0).all() and (dz[1] == 0).all()
    # rows with nothing to learn, or without weight in the sum, may hold anything
    z[9] = math.nan
    loss, stats = pnn.distill_loss(z, idx, t, y=y, temperature=2.0, alpha=0.25)
    z[1] = math.inf
    dz = pnn.distill_grad(z, idx, t, stats, g, y=y, temperature=2.0, alpha=0.25)
    assert loss[9] == 0 and (dz[9] == 0).all() and (dz[1] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,k", [(8, 12, 4), (8, 700, 40), (8, 9000, 9)])
def test_masked_classes(n, v, k, dtype):
    """Classes at -inf and at the type's lowest value; a row that a mask leaves nothing of; far-off logits; NaN."""
    z, idx, t, y, g = case(n, v, k, dtype, seed=7)
    low = torch.finfo(dtype).min
    masked = torch.rand(n, v, generator=torch.Generator().manual_seed(1)).cuda() < 0.5
    masked[torch.arange(n).cuda()[:, None], idx.long()] = False
    masked[torch.arange(n).cuda(), y.long()] = False
    for value in (-math.inf, low):
        zm = torch.where(masked, torch.tensor(value, dtype=dtype, device="cuda"), z)
        if value == low:
            zm[1] = low                        # all classes alike
        verify(zm, idx, t, y, g, 2.0, 0.25)
        verify(zm, idx, t, y, g, 1.0, 0.25)
    z2 = z.clone()
    z2[3] += 3e4                               # a large common offset (in bf16 it swallows the logits)
    z2[4] = -math.inf                          # nothing left
    loss, dz = verify(z2, idx, t, y, g, 2.0, 0.25)
    assert loss[4] == 0 and (dz[4] == 0).all()
    z2[5, 3] = math.nan
    z2[6] = math.nan
    loss, stats = pnn.distill_loss(z2, idx, t, y=y, temperature=2.0, alpha=0.25)
    dz = pnn.distill_grad(z2, idx, t, stats, g, y=y, temperature=2.0, alpha=0.25)
    assert torch.isnan(loss[5:7]).all() and torch.isnan(dz[5:7]).all()
    z3 = z.clone()
    z3[2, int(idx[2, 0])] = -math.inf          # the student excludes what the teacher gives weight
    loss, stats = pnn.distill_loss(z3, idx, t, temperature=2.0)
    dz = pnn.distill_grad(z3, idx, t, stats, temperature=2.0)
    assert loss[2] == math.inf and torch.isfinite(dz).all() and torch.isfinite(loss[[0, 1, 3, 4, 5, 6, 7]]).all()


@gpu
@pytest.mark.parametrize("n,v,k", [(16, 10, 3), (16, 300, 20), (3, 5000, 20)])
def test_gradient_against_differences(n, v, k):
    """Central differences of the loss in 64 bits of the same formula, at the classes with the largest slopes."""
    z, idx, t, y, g = case(n, v, k, F32, seed=9, scale=1.0)
    _, stats = pnn.distill_loss(z, idx, t, y=y, temperature=2.0, alpha=0.25)
    dz = pnn.distill_grad(z, idx, t, stats, y=y, temperature=2.0, alpha=0.25).double().cpu()
    one = torch.ones(n)
    for c in range(3):
        at = dz.abs().topk(3, dim=1).indices[:, c:c + 1]
        h = 1e-4
        up, down = (reference((z.double().cpu().scatter_add(1, at, torch.full((n, 1), s, dtype=torch.float64))), idx, t, y, 2.0,
                              0.25, one)[0] for s in (h, -h))
        # differences are off by h^2 / 6 of the third derivative (at most 1 here) and by 64-bit noise over h
        assert ((up - down) / (2 * h) - dz.gather(1, at)[:, 0]).abs().max() <= h * h + 1e-9 + 2.0 ** -20


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,k,pad", [(30, 10, 3, 0), (30, 500, 9, 3), (4, 10000, 30, 6)])
def test_gradient_in_place_and_strided(n, v, k, pad, dtype):
    z, idx, t, y, g = case(n, v, k, dtype, seed=11, pad=pad)
    loss, stats = pnn.distill_loss(z, idx, t, y=y, temperature=2.0, alpha=0.25)
    want = pnn.distill_grad(z, idx, t, stats, g, y=y, temperature=2.0, alpha=0.25)
    whole = torch.full((n + 2, v + 7), 5.0, dtype=dtype, device="cuda")
    plain = whole.clone()
    pnn.distill_grad(z, idx, t, stats, g, y=y, temperature=2.0, alpha=0.25, out=whole[1:-1, 3:-4])
    plain[1:-1, 3:-4] = want
    assert torch.equal(whole, plain)
    pnn.distill_grad(z, idx, t, stats, g, y=y, temperature=2.0, alpha=0.25, out=z)
    assert torch.equal(z, want)


@gpu
def test_rows_behind_32_bits():
    n, v = 20000, 110000
    z = torch.zeros(n, v, dtype=BF16, device="cuda")
    idx = torch.full((n, 2), -1, dtype=torch.int32, device="cuda")
    idx[-1, 0] = v - 1
    t = torch.zeros(n, 2, dtype=BF16, device="cuda")
    loss, stats = pnn.distill_loss(z, idx, t)
    dz = pnn.distill_grad(z, idx, t, stats, out=z)
    assert abs(float(loss[-1]) - math.log(v)) <= 1e-5 and (loss[:-1] == 0).all()
    assert float(dz[-1, -1]) == float(torch.tensor(1 / v - 1).to(BF16))
    assert (dz[-1, :-1] == torch.tensor(1 / v).to(BF16).cuda()).all() and (dz[:-1] == 0).all()


@gpu
@pytest.mark.parametrize("n,v,k", [(40, 10, 3), (4, 9000, 40)])
def test_another_stream_and_a_graph(n, v, k):
    z, idx, t, y, g = case(n, v, k, BF16)

    def step():
        loss, stats = pnn.distill_loss(z, idx, t, y=y, temperature=2.0, alpha=0.25)
        return loss, pnn.distill_grad(z, idx, t, stats, g, y=y, temperature=2.0, alpha=0.25)

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pnn.distill_loss(z, idx, t, y=y, temperature=2.0, alpha=0.25, stream=side)[0]
    side.synchronize()
    assert torch.equal(got, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for r in range(4):
        z.mul_(-0.75)
        y.copy_((y + 1) % v)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(kept, step()):
            assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v", [(30, 10), (30, 700), (5, 9000)])
def test_labels_alone(n, v, dtype):
    """alpha = 1 needs no teacher: the cross-entropy and its output error."""
    z, idx, t, y, g = case(n, v, 2, dtype, seed=13)
    loss, stats = pnn.distill_loss(z, None, None, y=y, alpha=1.0)
    dz = pnn.distill_grad(z, None, None, stats, g, y=y, alpha=1.0)
    want, tol, dwant, dtol = reference(z, idx, t, y, 1.0, 1.0, g)
    if dtype == BF16:
        dtol = dtol + (dwant.abs() + dtol) * torch.finfo(BF16).eps / 2
    assert ((loss.double().cpu() - want).abs() <= tol).all() and ((dz.double().cpu() - dwant).abs() <= dtol).all()
    loss, stats = pnn.distill_loss(z, None, None)  # neither a teacher nor labels
    assert (loss == 0).all() and (pnn.distill_grad(z, None, None, stats) == 0).all()


@gpu
def test_more_rows_than_one_launch_holds():
    n = (1 << 28) + 37  # 16 rows a workgroup of 256 threads, 2^32 threads
    z = torch.zeros(n, 2, device="cuda")
    z[:, 1] = 1
    y = torch.zeros(n, dtype=torch.int32, device="cuda")
    y[-1] = 1
    loss, stats = pnn.distill_loss(z, None, None, y=y, alpha=1.0)
    up = math.log1p(math.exp(1.0))
    assert abs(float(loss[0]) - up) <= 4e-7 and abs(float(loss[-2]) - up) <= 4e-7 and abs(float(loss[-1]) - (up - 1)) <= 4e-7
    assert float(loss.min()) == float(loss[-1]) and float(loss.max()) == float(loss[0])
    dz = pnn.distill_grad(z, None, None, stats, y=y, alpha=1.0, out=z)
    s = 1 / (1 + math.exp(1.0))
    assert abs(float(dz[0, 0]) - (s - 1)) <= 4e-7 and abs(float(dz[-1, 0]) - s) <= 4e-7
    assert (dz[:-1] == dz[0]).all()


@gpu
@pytest.mark.parametrize("dtype,n,v", [(F32, 4200, 8191), (BF16, 8400, 8190)])
def test_a_gradient_larger_than_the_caches(dtype, n, v):
    """Rows off 16 bytes with a ragged end; the entries' and the label's places are written after the rest of their row."""
    gen = torch.Generator(device="cuda").manual_seed(23)
    z = (torch.randn(n, v, generator=gen, device="cuda") * 3).to(dtype)
    idx = torch.randint(0, v, (n, 40), generator=gen, device="cuda", dtype=torch.int32)
    t = torch.randn(n, 40, generator=gen, device="cuda").to(dtype)
    y = torch.randint(0, v, (n,), generator=gen, device="cuda", dtype=torch.int32)
    g = torch.randn(n, generator=gen, device="cuda")
    assert 2 * z.numel() * z.element_size() > 256 << 20
    dz = torch.full_like(z, 7)
    loss, stats = pnn.distill_loss(z, idx, t, y=y, temperature=2.0, alpha=0.25)
    pnn.distill_grad(z, idx, t, stats, g, y=y, temperature=2.0, alpha=0.25, out=dz)
    at = torch.cat([torch.arange(8), torch.arange(n // 2, n // 2 + 8), torch.arange(n - 8, n)]).cuda()
    want, tol, dwant, dtol = reference(z[at], idx[at], t[at], y[at], 2.0, 0.25, g[at])
    if dtype == BF16:
        dtol = dtol + (dwant.abs() + dtol) * torch.finfo(BF16).eps / 2
    assert ((loss[at].double().cpu() - want).abs() <= tol).all() and ((dz[at].double().cpu() - dwant).abs() <= dtol).all()
    again = pnn.distill_grad(z, idx, t, stats, g, y=y, temperature=2.0, alpha=0.25, out=z)
    assert again is z and torch.equal(z, dz)  # in place
