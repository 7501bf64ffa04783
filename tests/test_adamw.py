"""The AdamW step over many tensors: values against the formulas in 64 bits, 8-bit states to the last bit and in the mean."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
FAKE = 1 << 20


# ---- refusals, on the host -----------------------------------------------------------------------

ARGS = dict(plan=FAKE, chunks=1, bits=32, g_type=pnn.FP32, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, lr_dev=None,
            seed=0, steps=FAKE)
TENSOR = dict(p=FAKE, g=FAKE, m=FAKE, v=FAKE, m_scale=None, v_scale=None, copy=None, n=10)


def planned(tensors=(TENSOR,), count=None, bits=32, g_type=pnn.FP32, plan=FAKE, size=1 << 20):
    t = (pnn.PnnAdamwTensor * max(1, len(tensors)))(*(pnn.PnnAdamwTensor(*d.values()) for d in tensors))
    return pnn.lib().pnn_adamw_plan(t, len(tensors) if count is None else count, bits, g_type, plan, size, None)


@pytest.mark.parametrize("over", [
    dict(plan=None), dict(plan=FAKE + 8), dict(chunks=-1), dict(chunks=1 << 31), dict(bits=16), dict(g_type=2), dict(lr=-1.0), dict(lr=math.nan),
    dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(beta2=1 - 1e-12), dict(eps=0.0),
    dict(eps=2.0), dict(eps=math.nan), dict(weight_decay=-1.0), dict(weight_decay=math.inf), dict(lr_dev=FAKE + 2), dict(steps=None),
    dict(steps=FAKE + 1)])
def test_steps_are_refused(over):
    a = pnn.PnnAdamw(*{**ARGS, **over}.values())
    assert pnn.lib().pnn_adamw_step(ctypes.byref(a), None) == pnn.PNN_EINVAL
    assert pnn.lib().pnn_last_error(None)


@pytest.mark.parametrize("over,status", [(dict(n=-1), pnn.PNN_ESHAPE), (dict(n=(1 << 40) + 1), pnn.PNN_ESHAPE)] + [
    (d, pnn.PNN_EINVAL) for d in (
        dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(p=FAKE + 2), dict(g=FAKE + 2), dict(m=FAKE + 1), dict(v=FAKE + 2),
        dict(copy=FAKE + 1))])
def test_tensors_are_refused(over, status):
    assert planned((TENSOR, {**TENSOR, **over})) == status
    assert pnn.lib().pnn_last_error(None)


def test_memory_is_refused():
    L, size, chunks = pnn.lib(), ctypes.c_int64(), ctypes.c_int64()
    assert L.pnn_adamw_step(None, None) == pnn.PNN_EINVAL
    assert planned(count=-1) == pnn.PNN_ESHAPE and planned(bits=16) == planned(g_type=2) == pnn.PNN_EINVAL
    assert planned(plan=None) == planned(plan=FAKE + 8) == pnn.PNN_EINVAL and planned(size=16) == pnn.PNN_ESHAPE
    assert L.pnn_adamw_plan(None, 1, 32, 0, FAKE, 1 << 20, None) == pnn.PNN_EINVAL
    assert planned(({**TENSOR, "n": 0, "p": None},), plan=None) == planned((), plan=None) == pnn.PNN_OK
    assert planned(({**TENSOR, "n": 1 << 40},) * 16) == pnn.PNN_ESHAPE
    t = (pnn.PnnAdamwTensor * 2)(*(pnn.PnnAdamwTensor(*{**TENSOR, "n": n}.values()) for n in (4097, 1)))
    assert L.pnn_adamw_bytes(t, 2, ctypes.byref(size), ctypes.byref(chunks)) == pnn.PNN_OK and chunks.value == 3 and size.value >= 3 * 56
    assert L.pnn_adamw_bytes(t, 2, None, ctypes.byref(chunks)) == L.pnn_adamw_bytes(t, 2, ctypes.byref(size), None) == pnn.PNN_EINVAL
    for over in (dict(), dict(m_scale=FAKE), dict(m_scale=FAKE + 2, v_scale=FAKE), dict(m_scale=FAKE, v_scale=FAKE + 2)):
        assert planned(({**TENSOR, **over},), bits=8) == pnn.PNN_EINVAL
    good = [FAKE, FAKE, FAKE, FAKE, 10, FAKE, FAKE]
    for i, value, status in [(i, None, pnn.PNN_EINVAL) for i in (0, 1, 2, 3, 5, 6)] + [(i, FAKE + 2, pnn.PNN_EINVAL) for i in (2, 3, 5, 6)] + [
            (4, -1, pnn.PNN_ESHAPE), (4, (1 << 40) + 1, pnn.PNN_ESHAPE), (4, 0, pnn.PNN_OK)]:
        assert L.pnn_adamw_values(*(value if j == i else x for j, x in enumerate(good)), None) == status


def test_the_binding_refuses():
    def p(*shape, dtype=F32):
        return torch.zeros(*shape, dtype=dtype)

    for a, kw, why in (
            (([], []), {}, "no parameters"), (([p(3)], [p(3)]), dict(bits=16), "bits"), (([p(3)], []), {}, "as many"),
            (([p(3)], [p(3)]), dict(copies=[]), "as many"), (([p(3)], [p(4)]), {}, "grads"), (([p(3, dtype=BF16)], [p(3)]), {}, "params"),
            (([p(3)] * 1 + [p(2)], [p(3), p(2, dtype=BF16)]), {}, "grads"), (([p(4, 3).T], [p(3, 4)]), {}, "contiguous"),
            (([p(3)], [p(3)]), dict(copies=[p(3)]), "copies"), (([p(3)], [p(3)]), dict(state=[[p(3)]]), "state"),
            (([p(3)], [p(3)]), dict(state=[[p(3)], [p(2)]]), "v"), (([p(3)], [p(3)]), dict(bits=8, state=[[p(3)], [p(3)]]), "state"),
            (([p(3)], [p(3)]), dict(steps=torch.zeros(1, dtype=torch.int32)), "steps"), (([p(3)], [p(3)]), dict(lr=torch.zeros(2)), "lr"),
            (([p(3)], [p(3, dtype=torch.float64)]), {}, "float32 or bfloat16")):
        with pytest.raises(ValueError, match=why):
            pnn.AdamW(*a, **kw)
    one = p(5)
    for a, kw in (([one, one], {}), ([one[:3], one[2:]], {}), ([one], dict(state=[[one], [p(5)]])), ([one[:2]], dict(copies=[one.view(BF16)[3:5]]))):
        with pytest.raises(ValueError, match="overlap"):
            pnn.AdamW(a, [torch.zeros_like(x) for x in a], **kw)
    with pytest.raises(ValueError, match="CUDA"):
        pnn.AdamW([one[:2], one[2:], one[5:]], [p(2), p(3), p(0)])
    with pytest.raises(ValueError, match="CUDA"):
        pnn.AdamW([p(3)], [p(3)])
    with pytest.raises(ValueError, match="m is"):
        pnn.adamw_values(p(3), p(3), p(1), p(1)) if torch.cuda.is_available() else pnn._values(p(3), "m", (3,), torch.uint8)


# ---- what a code stands for, and which code a value gets -----------------------------------------

def level(c, top):
    """Values of codes without their scale, fp32 (a power of two's root rounded once)."""
    c = np.asarray(c, dtype=np.int64)
    return np.where(c > 0, np.exp2((c - top) / 8.0), 0.0).astype(np.float32)


def mix(x):
    x = np.asarray(x, dtype=np.uint64) & np.uint64(0xFFFFFFFF)
    for shift, by in ((16, 0x6A09E667), (15, 0xBB67AE85)):
        x ^= x >> np.uint64(shift)
        x = (x * np.uint64(by)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def bits_of(seed, step, tensor, n):
    at = np.arange(n, dtype=np.uint64)
    key = mix(mix(mix(seed + 0x6A09E667 * step) + np.uint64(tensor)) + at // np.uint64(256))
    return mix(key + at % np.uint64(256))


def codes_of(x, top, lowest, u):
    """Codes and scales of sizes x (fp32), block by block: the two levels about a value by a search, and the share."""
    code = np.zeros(len(x), dtype=np.uint8)
    scales = np.zeros(-(-len(x) // 256), dtype=np.float32)
    for b in range(len(scales)):
        at = slice(256 * b, min(len(x), 256 * b + 256))
        y = x[at]
        scale = scales[b] = y.max() if np.isfinite(y).all() else np.float32(np.nan)
        if not scale > 0:
            continue
        grid = level(np.arange(top + 1), top) * scale  # (fp32)
        c = np.searchsorted(grid, y, side="right") - 1
        above = grid[np.minimum(c + 1, top)]
        up = (c < top) & (u[at] * (above - grid[c]) < y - grid[c])
        code[at] = np.where(y > 0, np.maximum(c + up, lowest), 0)
    return code, scales


def moments(g, m, v, betas):
    """The new moments in fp32, each operation rounded."""
    b1, c1, b2, c2 = (np.float32(x) for x in (betas[0], 1.0 - betas[0], betas[1], 1.0 - betas[1]))
    return b1 * m + c1 * g, b2 * v + c2 * g * g


# ---- values --------------------------------------------------------------------------------------

def reference(p, g, m, v, t, lr, betas, eps, decay):
    """p, m, v after step t in 64 bits, and what they may be off by."""
    p, g, m, v = (x.double().cpu() for x in (p, g, m, v))
    m1, v1 = betas[0] * m + (1 - betas[0]) * g, betas[1] * v + (1 - betas[1]) * g * g
    # a factor's rounding, a product's, the sum's
    moff = 2 * U * (betas[0] * m.abs() + (1 - betas[0]) * g.abs()) + U * m1.abs() + 2.0 ** -149
    voff = 5 * U * v1 + 2.0 ** -148
    step, root = lr / (1 - betas[0] ** t), 1 / (1 - betas[1] ** t)
    low = (v1 * root).sqrt() + eps
    out = p * (1 - lr * decay) - step * m1 / low
    # the rates (rounded, logarithm and expm1: eight half steps), root and quotient
    off = 4 * U * p.abs() + step / low * (moff + 20 * U * m1.abs()) + 2 * U * out.abs()
    return (out, off), (m1, moff), (v1, voff)


def tensors(sizes, grads=F32, seed=0, at=0):
    g = torch.Generator().manual_seed(seed)

    def part(n, dtype=F32, scale=1.0):  # (`at` values off the start of an allocation)
        return (torch.randn(n + at, generator=g) * scale).to(dtype).cuda()[at:]

    p = [part(n, scale=0.1) for n in sizes]
    gr = [(part(n) * torch.exp(2 * part(n))).to(grads) for n in sizes]
    return p, gr, [part(n, scale=0.3) for n in sizes], [part(n).square() + 1e-3 for n in sizes]


HYPER = dict(lr=1e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1)
SIZES = [[1], [3, 256, 257, 10, 4096, 4097, 0, 100001], list(range(1, 131)), [4095] * 50]


def near(got, want, off):
    got = got.double().cpu()
    ok = (got - want).abs() <= off
    assert ok.all(), f"{int((~ok).sum())} of {ok.numel()}, largest {((got - want).abs() / off)[~ok].max():.3g} of the tolerance"


@gpu
@pytest.mark.parametrize("grads", [F32, BF16])
@pytest.mark.parametrize("at", [0, 1])
@pytest.mark.parametrize("sizes", SIZES)
def test_a_step(sizes, at, grads):
    p, g, m, v = tensors(sizes, grads, at=at)
    copies = [torch.zeros(n + at, dtype=BF16, device="cuda")[at:] if i % 3 != 1 else None for i, n in enumerate(sizes)]
    for t in (1, 7, 100000):
        want = [reference(a, b, c, d, t, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"]) for a, b, c, d in zip(p, g, m, v)]
        steps = torch.tensor([t - 1, 0], dtype=torch.int32, device="cuda")
        opt = pnn.AdamW(p, g, copies=copies, state=[m, v], steps=steps, **HYPER)
        opt.step()
        assert steps.tolist() == [t, 0]
        for a, c, d, q, w in zip(p, m, v, copies, want):
            near(a, *w[0])
            near(c, *w[1])
            near(d, *w[2])
            assert q is None or torch.equal(q, a.to(BF16))


@gpu
@pytest.mark.parametrize("grads", [F32, BF16])
@pytest.mark.parametrize("at", [0, 1])
@pytest.mark.parametrize("sizes", SIZES)
def test_steps_in_8_bits(sizes, at, grads):
    """Three steps from zeros: each step's parameters from the states that the codes stand for, its codes to the bit."""
    p, g, _, _ = tensors(sizes, grads, seed=1, at=at)
    codes = [[torch.zeros(n + at, dtype=torch.uint8, device="cuda")[at:] for n in sizes] for _ in range(2)]
    scales = [[torch.zeros(-(-n // 256), device="cuda") for n in sizes] for _ in range(2)]
    opt = pnn.AdamW(p, g, bits=8, state=codes + scales, seed=99, **HYPER)
    for t in (1, 2, 3):
        held = [pnn.adamw_values(*x) for x in zip(*opt.state)]
        want = [reference(a, b, *c, t, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"]) for a, b, c in zip(p, g, held)]
        opt.step()
        for i, n in enumerate(sizes):
            near(p[i], *want[i][0])
            m, v = moments(g[i].float().cpu().numpy(), held[i][0].cpu().numpy(), held[i][1].cpu().numpy(), HYPER["betas"])
            bits = bits_of(99, t, i, n)
            um, uv = (((b.astype(np.float32) + np.float32(0.5)) / np.float32(65536)) for b in (bits >> np.uint64(16), bits & np.uint64(0xFFFF)))
            cm, sm = codes_of(np.abs(m), 127, 0, um)
            cv, sv = codes_of(v, 255, 1, uv)
            got = [x[i].cpu().numpy() for x in opt.state]
            assert np.array_equal(got[2], sm) and np.array_equal(got[3], sv)
            assert np.array_equal(got[0], cm | np.where(m < 0, 128, 0).astype(np.uint8)) and np.array_equal(got[1], cv)
            vm, vv = (x.cpu().numpy() for x in pnn.adamw_values(*(x[i] for x in opt.state)))
            at_block = np.arange(n) // 256
            assert np.array_equal(vm, np.where(m < 0, -1, 1).astype(np.float32) * level(cm, 127) * sm[at_block])
            assert np.array_equal(vv, level(cv, 255) * sv[at_block])
        for x in g:
            x.mul_(-0.5)
    assert opt.steps.tolist() == [3, 0]


@gpu
def test_rounding_is_right_in_the_mean():
    """Values of many sizes, a million times each: the mean of what is kept is the value (a level is at most 9.1 % wide:
    a rounding's deviation is at most half of that, the mean's a 1,000th, and six of those are allowed)."""
    n = 256 * 4096
    sizes = np.exp2(-np.linspace(0, 14.5, 256)).astype(np.float32)
    g = torch.from_numpy(np.tile(sizes, n // 256)).cuda()
    opt = pnn.AdamW([torch.zeros(n, device="cuda")], [g], bits=8, betas=(0.5, 0.5), seed=3)
    opt.step()
    m, v = pnn.adamw_values(*(s[0] for s in opt.state))
    for got, want in ((m, 0.5 * sizes.astype(np.float64)), (v, 0.5 * sizes.astype(np.float64) ** 2)):
        mean = got.view(-1, 256).double().mean(0).cpu().numpy()
        assert (np.abs(mean / want - 1) <= 6 * 0.5 * 0.0906 / math.sqrt(4096)).all()
    # m and v, neighbours and blocks are rounded apart
    up = (m.view(-1, 256).double().cpu() > torch.from_numpy(0.5 * sizes.astype(np.float64))).double()
    both = [up[:, 1:] * up[:, :-1], up[1:] * up[:-1], up * (v.view(-1, 256).double().cpu() > torch.from_numpy(0.5 * sizes.astype(np.float64) ** 2))]
    share = up.mean(0)
    other = (v.view(-1, 256).double().cpu() > torch.from_numpy(0.5 * sizes.astype(np.float64) ** 2)).double().mean(0)
    for got, alone in zip(both, (share[1:] * share[:-1], share * share, share * other)):
        assert (got.mean(0) - alone).abs().max() <= 6 * 0.5 / math.sqrt(4096)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_extremes(bits):
    """Gradients of zero, far too small and too large, infinities and NaN: they reach their own values, or their block."""
    n = 256 * 6
    g = torch.ones(n, device="cuda")
    g[:256] = 0                                # never a gradient: the parameters only decay
    g[256:512] = 1e-25                         # squares below the range of fp32
    g[300] = 0
    g[512:768] = 1e25                          # squares beyond it
    g[768 + 5] = math.nan
    g[1024 + 5] = math.inf
    p = torch.full((n,), 0.5, device="cuda")
    opt = pnn.AdamW([p], [g], bits=bits, **HYPER)
    for t in (1, 2):
        opt.step()
        m, v = opt.state[0][0], opt.state[1][0]
        if bits == 8:
            m, v = pnn.adamw_values(*(s[0] for s in opt.state))
        assert (p[:256] == p[0]).all() and abs(float(p[0]) - 0.5 * 0.999 ** t) <= 4 * U and (m[:256] == 0).all() and (v[:256] == 0).all()
        assert torch.isfinite(p[256:512]).all() and torch.isfinite(m[256:512]).all() and m[300] == 0
        if t == 1:
            assert (p[512:768] == p[0]).all()  # (an infinite root: no step)
            for block in (3, 4):
                rest = torch.arange(256, device="cuda") != 5
                assert torch.isfinite(p[256 * block:][:256][rest]).all()
                assert not torch.isfinite(p[256 * block + 5])
                if bits == 32:
                    assert torch.isfinite(m[256 * block:][:256][rest]).all() and torch.isfinite(v[256 * block:][:256][rest]).all()
                else:
                    assert torch.isnan(m[256 * block:][:256]).all() and torch.isnan(v[256 * block:][:256]).all()
        assert torch.isfinite(p[1280:]).all() and torch.isfinite(m[1280:]).all() and torch.isfinite(v[1280:]).all()
        assert (v[1280:] > 0).all()


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_the_last_values_of_a_tensor_behind_32_bits(bits):
    n = (1 << 32) + 300
    p = torch.zeros(n, device="cuda")
    g = torch.zeros(n, dtype=BF16, device="cuda")
    p[-300:], g[-300:], g[:2], p[-301] = 1, 2, -2, 1
    opt = pnn.AdamW([p], [g], bits=bits, lr=0.5, weight_decay=0.0)
    opt.step()
    # the first step is the rate, whatever the gradient
    assert (p[-300:] - 0.5).abs().max() <= 2e-6 and float(p[-301]) == 1 and (p[:2] - 0.5).abs().max() <= 2e-6
    assert int(torch.count_nonzero(p[2:-301])) == 0
    assert int(torch.count_nonzero(opt.state[0][0])) == 302 and (opt.state[0][0][-300:] != 0).all()


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_what_lies_beside_a_tensor_is_left(bits):
    """Tensors in one memory, a few values apart: a step writes its tensors' values alone."""
    sizes = [5, 300, 1, 4100]
    arenas = []

    def parts(dtype, fill, per=1):
        total = sum(-(-n // per) + 3 for n in sizes)
        arenas.append((torch.full((total,), fill, dtype=dtype, device="cuda"), per))
        at = 0
        out = []
        for n in sizes:
            out.append(arenas[-1][0][at + 1:at + 1 + -(-n // per)])
            at += -(-n // per) + 3
        return out

    p, g, copies = parts(F32, 7.0), parts(F32, 7.0), parts(BF16, 7.0)
    state = [parts(F32, 7.0), parts(F32, 7.0)] if bits == 32 else [parts(torch.uint8, 7), parts(torch.uint8, 7), parts(F32, 7.0, 256), parts(F32, 7.0, 256)]
    pnn.AdamW(p, g, copies=copies, bits=bits, state=state).step()
    for arena, per in arenas:
        outside, at = torch.ones(arena.numel(), dtype=torch.bool), 0
        for n in sizes:
            outside[at + 1:at + 1 + -(-n // per)] = False
            at += -(-n // per) + 3
        assert (arena.cpu()[outside] == 7).all()
    assert all((x != 7).all() for x in p)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_graph_another_stream_and_resumed_training(bits):
    sizes = [300] * 60 + [5000]  # (two launches)
    first = tensors(sizes, seed=5)
    g = first[1]

    def fresh(lr):
        p = [x.clone() for x in first[0]]
        return p, pnn.AdamW(p, g, bits=bits, lr=lr, betas=(0.9, 0.99), seed=11, copies=[x.to(BF16) for x in p])

    def same(a, b):
        return all(torch.equal(x, y) for x, y in zip(a.params + a.copies + sum(a.state, []) + [a.steps], b.params + b.copies + sum(b.state, []) + [b.steps]))

    rate = torch.tensor([0.01], device="cuda")
    _, eager = fresh(0.01)
    _, other = fresh(rate)
    _, recorded = fresh(rate)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded.step()
    for r in range(5):
        eager.lr = 0.01 / (r + 1)
        rate.fill_(0.01 / (r + 1))
        eager.step()
        side.wait_stream(torch.cuda.current_stream())
        other.step(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        graph.replay()
        torch.cuda.synchronize()
        assert same(eager, other) and same(eager, recorded) and eager.steps.tolist() == [r + 1, 0]
        if r == 2:  # saved and taken up again
            copy = [[x.clone() for x in s] for s in eager.state]
            p = [x.clone() for x in eager.params]
            again = pnn.AdamW(p, g, bits=bits, lr=0.01, betas=(0.9, 0.99), seed=11, copies=[x.to(BF16) for x in p], state=copy, steps=eager.steps.clone())
        if r > 2:
            again.lr = 0.01 / (r + 1)
            again.step()
            assert same(eager, again)
        for x in g:
            x.mul_(-0.75)
    assert other.lr is rate
    with pytest.raises(ValueError, match="tensor"):
        other.lr = 0.1


@gpu
def test_no_values_still_count():
    opt = pnn.AdamW([torch.zeros(0, device="cuda")], [torch.zeros(0, device="cuda")])
    opt.step()
    opt.step()
    assert opt.steps.tolist() == [2, 0]


@gpu
def test_a_step_follows_the_difference_of_the_loss():
    """Betas of 0: the step is the gradient's sign by its size over the root of its square, lr for every value."""
    p, g, _, _ = tensors([1000], seed=9)
    before = p[0].clone()
    pnn.AdamW(p, g, betas=(0.0, 0.0), lr=0.25, weight_decay=0.0, eps=1e-20).step()
    assert (p[0] - (before - 0.25 * torch.sign(g[0]))).abs().max() <= 8 * U
