"""A handle's child networks on rows that name them: answers and training steps against the formulas in
64 bits, the two chained as a program uses them (a step of the CNs towards the answers of others), and
against the calls on slices."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu
F64 = torch.float64


def test_null_handles_are_refused():
    L = pnn.lib()
    assert L.pnn_infer_routed(None, None, 4, None, 1, None, None, None, None) == pnn.PNN_EINVAL
    assert L.pnn_train_routed(None, None, 4, None, 1, None, None, 0, None, 1.0, 0.0, None, None) == pnn.PNN_EINVAL


def network(sizes, acts, replicas, precision=pnn.FP32, lr=0.5, batch=4, loss=pnn.LOSS_XENT, seed=1):
    cfg = pnn.make_config(sizes, acts, loss, precision, replicas, batch, lr)
    g = np.random.default_rng(seed)
    net = pnn.PNN(cfg, np.zeros(pnn.param_count(cfg), np.float32))
    for k in range(replicas):  # CNs that differ
        parts = []
        for i, o in zip(sizes, sizes[1:]):
            parts += [g.uniform(-1, 1, i * o) * math.sqrt(6 / (i + o)), g.normal(0, 0.1, o)]
        net.set_params(k, np.concatenate(parts).astype(np.float32))
    return net


def layers(net, k):
    flat, out, o = torch.from_numpy(net.get_params(k)).to(F64), [], 0
    s = list(net.cfg.sizes)[:net.cfg.n_layers + 1]
    for i, j in zip(s, s[1:]):
        out.append((flat[o:o + i * j].view(j, i).clone(), flat[o + i * j:o + i * j + j].clone()))
        o += i * j + j
    return out


def rounded(t, net):
    return t.to(torch.bfloat16).to(F64) if net.cfg.precision == pnn.BF16_MIXED else t


def phi(act, z):
    return {pnn.SIGMOID: torch.sigmoid, pnn.TANH: torch.tanh, pnn.RELU: lambda v: torch.where(v < 0, -0.0, v),
            pnn.LEAKY_RELU: lambda v: torch.where(v < 0, 0.01 * v, v)}[act](z)


def slope(act, a):
    neg = torch.signbit(a)
    return {pnn.SIGMOID: a * (1 - a), pnn.TANH: 1 - a * a, pnn.RELU: torch.where(neg, 0.0, 1.0).to(F64),
            pnn.LEAKY_RELU: torch.where(neg, 0.01, 1.0).to(F64)}[act]


def forward(net, params, x):
    """The activations that enter each layer's product, and the last layer's sums."""
    a = [rounded(x, net)]
    for l, (w, b) in enumerate(params):
        z = a[-1] @ rounded(w, net).T + b
        if l < len(params) - 1:
            a.append(rounded(phi(net.cfg.act[l], z), net))
    return a, z


def answers(net, x, ids, weights):
    n, per_row = ids.shape
    out, count = torch.zeros(n, net.cfg.sizes[net.cfg.n_layers], dtype=F64), torch.zeros(n, 1, dtype=F64)
    for k in range(net.K):
        _, z = forward(net, layers(net, k), x)
        act = net.cfg.act[net.cfg.n_layers - 1]
        o = torch.softmax(z, 1) if act == pnn.SOFTMAX else phi(act, z)
        for j in range(per_row):
            hit = (ids[:, j] == k).to(F64)[:, None]
            out += o * hit * (weights[:, j:j + 1] if weights is not None else 1.0)
            count += hit
    return (out if weights is not None else out / count.clamp(min=1)), count[:, 0] > 0


def step(net, params, x, idx, t, y, temperature, alpha):
    """New parameters of one CN, and the losses, for the rows x that name it."""
    a, z = forward(net, params, x)
    q, s = torch.softmax(z / temperature, 1), torch.softmax(z, 1)
    loss, d = torch.zeros(len(x), dtype=F64), torch.zeros_like(z)
    if idx is not None and alpha < 1:
        kept = (idx >= 0) & (idx < z.shape[1])
        p = torch.softmax(torch.where(kept, t / temperature, -math.inf), 1)
        at = torch.where(kept, idx, 0)
        p = torch.where(kept & kept.any(1, keepdim=True), p, 0.0)
        some = kept.any(1)
        kl = torch.where(p > 0, p * (torch.log(p) - torch.log(q.gather(1, at))), 0.0).sum(1)
        loss += (1 - alpha) * temperature ** 2 * kl
        d += (1 - alpha) * temperature * (q * some[:, None] - torch.zeros_like(z).scatter_add(1, at, p))
    if y is not None and alpha > 0:
        some = (y >= 0) & (y < z.shape[1])
        yc = torch.where(some, y, 0)[:, None]
        loss += torch.where(some, -alpha * torch.log(s.gather(1, yc))[:, 0], 0.0)
        d += alpha * (s - torch.zeros_like(z).scatter(1, yc, 1.0)) * some[:, None]
    d, new = rounded(d, net), [None] * len(params)
    for l in range(len(params) - 1, -1, -1):
        w, b = params[l]
        eta = float(np.float32(net.cfg.lr)) / len(x)
        new[l] = (w - eta * d.T @ a[l], b - eta * d.sum(0))
        if l:
            d = rounded((d @ rounded(w, net)) * slope(net.cfg.act[l - 1], a[l]), net)
    return new, loss


def batch(n, per_row, net, seed, top=3, drop=0.1):
    g = torch.Generator().manual_seed(seed)
    x = torch.rand(n, net.cfg.sizes[0], generator=g)
    ids = torch.randint(0, net.K, (n, per_row), generator=g, dtype=torch.int32)
    ids[torch.rand(n, per_row, generator=g) < drop] = -1
    o = net.cfg.sizes[net.cfg.n_layers]
    idx = torch.stack([torch.randperm(o, generator=g)[:top] for _ in range(n)]).to(torch.int32)
    idx[torch.rand(n, top, generator=g) < 0.1] = -1
    t = torch.randn(n, top, generator=g) * 2
    y = torch.randint(-1, o, (n,), generator=g, dtype=torch.int32)
    return x, ids, idx, t, y


NETS = [((784, 16, 10), (pnn.SIGMOID, pnn.SOFTMAX), 1, pnn.FP32), ((48, 40, 24, 10), (pnn.RELU, pnn.TANH, pnn.SOFTMAX), 5, pnn.FP32),
        ((32, 10), (pnn.SOFTMAX,), 3, pnn.FP32), ((784, 256, 10), (pnn.RELU, pnn.SOFTMAX), 4, pnn.BF16_MIXED),
        ((64, 32, 16), (pnn.LEAKY_RELU, pnn.SOFTMAX), 70, pnn.BF16_MIXED)]


@gpu
@pytest.mark.parametrize("n,per_row", [(1, 1), (37, 2), (900, 1), (300, 3)])
@pytest.mark.parametrize("sizes,acts,replicas,precision", NETS)
def test_answers(sizes, acts, replicas, precision, n, per_row):
    net = network(sizes, acts, replicas, precision)
    x, ids, _, _, _ = batch(n, per_row, net, 3)
    w = torch.rand(n, per_row)
    for weights in (None, w):
        want, some = answers(net, x.to(F64), ids, None if weights is None else weights.to(F64))
        pred = torch.empty(n, dtype=torch.int32, device="cuda")
        out = torch.empty(n, sizes[-1], device="cuda")
        net.infer_routed(x.cuda(), ids.cuda(), pred, None if weights is None else w.cuda(), out)
        # (a bf16 activation on the other side of a rounding moves an output by a step of its share)
        assert (out.cpu().to(F64) - want).abs().max() <= (2e-2 if precision else 1e-5) * per_row
        assert torch.equal(pred.cpu()[some], out.cpu().argmax(1).to(torch.int32)[some])
        assert (pred.cpu()[~some] == -1).all() and (out.cpu()[~some] == 0).all()
        again = torch.empty_like(pred)
        net.infer_routed(x.cuda(), ids.cuda(), again, None if weights is None else w.cuda())
        assert torch.equal(again, pred)


@gpu
def test_answers_of_one_network_are_those_of_infer():
    net = network((784, 128, 10), (pnn.SIGMOID, pnn.SIGMOID), 4, loss=pnn.LOSS_MSE)
    x = torch.rand(70000, 784, device="cuda")  # more than one chunk
    ids = torch.full((70000, 1), 2, dtype=torch.int32, device="cuda")
    got, want = (torch.empty(70000, 10, device="cuda") for _ in range(2))
    pred = torch.empty(70000, dtype=torch.int32, device="cuda")
    net.infer_routed(x, ids, pred, out=got)
    net.infer(x, pred, which=2, out=want)
    assert (got - want).abs().max() <= 1e-5


def parity(got, ref):
    floor = ref.pow(2).mean().sqrt()
    return ((got - ref).abs() / torch.maximum(ref.abs(), floor)).max()


@gpu
@pytest.mark.parametrize("n,per_row", [(1, 1), (37, 2), (900, 1), (300, 3)])
@pytest.mark.parametrize("sizes,acts,replicas,precision", NETS)
def test_training_steps(sizes, acts, replicas, precision, n, per_row):
    """Each step starts from the library's own parameters: every weight within the suite's bars of one step
    (1e-5 in fp32, 2e-2 in bf16-mixed), and what the step added within 1e-3 (1e-2) of its own norm per layer."""
    net = network(sizes, acts, replicas, precision)
    merged = net.get_params(-1)
    for r, (temperature, alpha) in enumerate(((2.0, 0.25), (1.0, 1.0), (3.0, 0.0))):
        x, ids, idx, t, y = batch(n, per_row, net, 10 + r)
        before = [layers(net, k) for k in range(net.K)]
        loss = torch.empty(n, per_row, device="cuda")
        net.train_routed(x.cuda(), ids.cuda(), idx.cuda(), t.cuda(), y.cuda() if alpha else None, temperature, alpha, loss)
        want_loss = torch.zeros(n * per_row, dtype=F64)
        for k in range(net.K):
            members = torch.nonzero(ids.reshape(-1) == k)[:, 0]
            rows, after = members // per_row, layers(net, k)
            if len(rows) == 0:
                assert all(torch.equal(a, b) for p, q in zip(after, before[k]) for a, b in zip(p, q))
                continue
            want, want_loss[members] = step(net, before[k], x[rows].to(F64), idx[rows].long(), t[rows].to(F64), y[rows].long(),
                                            temperature, alpha)
            for (w, b), (wr, br), (w0, b0) in zip(after, want, before[k]):
                assert parity(w, wr) <= (2e-2 if precision else 1e-5) and parity(b, br) <= (2e-2 if precision else 1e-5)
                moved, added = torch.cat([(wr - w0).flatten(), br - b0]), torch.cat([(w - w0).flatten(), b - b0])
                # (stored parameters are rounded to fp32: half a step of each)
                held = 2.0 ** -24 * torch.cat([w0.flatten(), b0]).norm()
                assert (added - moved).norm() <= (1e-2 if precision else 1e-3) * moved.norm() + held
        assert (loss.reshape(-1).cpu().to(F64) - want_loss).abs().max() <= (2e-1 if precision else 1e-4)
        assert (loss.reshape(-1).cpu()[ids.reshape(-1) < 0] == 0).all()
    assert np.array_equal(net.get_params(-1), merged)


@gpu
@pytest.mark.parametrize("batch_size", [64, 128])
def test_a_step_on_slices_is_the_step_of_train_epoch(batch_size):
    """Labels alone and rows that name the CN of their slice; CNs as a deferred broadcast left them."""
    sizes, acts, K = (784, 256, 10), (pnn.SIGMOID, pnn.SOFTMAX), 4
    a, b = (network(sizes, acts, K, batch=batch_size, lr=0.1) for _ in range(2))
    for net in (a, b):
        net.merge(broadcast=True)
    n = batch_size * K
    x = torch.rand(n, 784, device="cuda")
    y = torch.randint(0, 10, (n,), device="cuda", dtype=torch.int32)
    ids = torch.arange(K, dtype=torch.int32, device="cuda").repeat_interleave(batch_size)[:, None].contiguous()
    a.train_epoch(x, y)
    b.train_routed(x, ids, y=y, alpha=1.0)
    for k in range(K):
        assert parity(torch.from_numpy(b.get_params(k)), torch.from_numpy(a.get_params(k))) <= 1e-5


@gpu
def test_networks_learn_from_the_answers_of_others():
    """The chain: combined answers of four CNs, their top three classes as the teacher, one more CN as the student."""
    net = network((64, 48, 10), (pnn.TANH, pnn.SOFTMAX), 5)
    n = 400
    x = torch.rand(n, 64, device="cuda")
    teachers = torch.arange(4, dtype=torch.int32, device="cuda").repeat(n, 1)
    student = torch.full((n, 1), 4, dtype=torch.int32, device="cuda")
    pred = torch.empty(n, dtype=torch.int32, device="cuda")
    out, loss = torch.empty(n, 10, device="cuda"), torch.empty(n, 1, device="cuda")
    net.infer_routed(x, teachers, pred, out=out)
    top = out.topk(3, dim=1)
    idx, t = top.indices.to(torch.int32), top.values.log()
    before, others = layers(net, 4), [net.get_params(k) for k in range(4)]
    net.train_routed(x, student, idx, t, loss=loss)
    want, want_loss = step(net, before, x.cpu().to(F64), idx.cpu().long(), t.cpu().to(F64), None, 1.0, 0.0)
    for (w, b), (wr, br) in zip(layers(net, 4), want):
        assert parity(w, wr) <= 1e-5 and parity(b, br) <= 1e-5
    assert (loss[:, 0].cpu().to(F64) - want_loss).abs().max() <= 1e-4
    assert all(np.array_equal(net.get_params(k), o) for k, o in enumerate(others))
    # its gradient, through the parameters: the losses' sum falls along the step by its squared norm
    eta = net.cfg.lr / n
    moved = sum(float(((w - w0) / -eta).pow(2).sum() + ((b - b0) / -eta).pow(2).sum()) for (w, b), (w0, b0) in zip(layers(net, 4), before))
    h = 1e-3 / math.sqrt(moved)
    sides = []
    for s in (h, -h):
        p = [(w0 + (w - w0) / -eta * s, b0 + (b - b0) / -eta * s) for (w, b), (w0, b0) in zip(layers(net, 4), before)]
        sides.append(float(step(net, p, x.cpu().to(F64), idx.cpu().long(), t.cpu().to(F64), None, 1.0, 0.0)[1].sum()))
    assert abs((sides[0] - sides[1]) / (2 * h) - moved) <= 1e-3 * moved


@gpu
@pytest.mark.parametrize("precision", [pnn.FP32, pnn.BF16_MIXED])
def test_recorded_calls(precision):
    """A recorded answer and step replayed between eager work; a workspace cannot grow while recording, and one
    that a graph uses survives larger calls."""
    sizes, acts = (48, 40, 10), (pnn.RELU, pnn.SOFTMAX)
    eager, net = (network(sizes, acts, 3, precision) for _ in range(2))
    x, ids, idx, t, y = (v.cuda() for v in batch(60, 2, net, 5))
    pred, out, pred2, out2 = (torch.empty(60, *s, dtype=d, device="cuda") for s, d in
                              (((), torch.int32), ((10,), torch.float32)) * 2)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(pnn.PnnError) as e:
        with torch.cuda.graph(graph):
            net.infer_routed(x, ids, pred, out=out)
    assert e.value.status == pnn.PNN_EHIP
    saved = [net.get_params(k) for k in range(3)]
    net.infer_routed(x, ids, pred, out=out)
    net.train_routed(x, ids, idx, t, y, 2.0, 0.5)
    for k in range(3):
        net.set_params(k, saved[k])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.infer_routed(x, ids, pred, out=out)
        net.train_routed(x, ids, idx, t, y, 2.0, 0.5)
    for r in range(4):
        v = batch(60, 2, net, 60 + r)
        for a, b in zip((x, ids, idx, t, y), v):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        eager.infer_routed(x, ids, pred2, out=out2)
        eager.train_routed(x, ids, idx, t, y, 2.0, 0.5)
        assert torch.equal(pred, pred2) and torch.equal(out, out2)
        for k in range(3):
            assert np.array_equal(net.get_params(k), eager.get_params(k))
        if r == 1:  # a larger call replaces the workspace; the graph keeps its own
            big = batch(5000, 2, net, 70)
            big_pred = torch.empty(5000, dtype=torch.int32, device="cuda")
            net.infer_routed(big[0].cuda(), big[1].cuda(), big_pred)


@gpu
def test_refusals():
    net = network((16, 10), (pnn.SIGMOID,), 3, loss=pnn.LOSS_MSE)
    soft = network((16, 10), (pnn.SOFTMAX,), 3)
    x, ids, idx, t, y = (v.cuda() for v in batch(8, 2, soft, 1))
    pred = torch.empty(8, dtype=torch.int32, device="cuda")
    L = pnn.lib()

    def infer(h=net.h, x=x.data_ptr(), n=8, ids=ids.data_ptr(), per_row=2, pred=pred.data_ptr()):
        return L.pnn_infer_routed(h, x, n, ids, per_row, None, pred, None, None)

    def train(h=soft.h, x=x.data_ptr(), n=8, ids=ids.data_ptr(), per_row=2, idx=idx.data_ptr(), t=t.data_ptr(), top=3,
              y=y.data_ptr(), temperature=2.0, alpha=0.5):
        return L.pnn_train_routed(h, x, n, ids, per_row, idx, t, top, y, temperature, alpha, None, None)

    for call in (lambda: infer(x=None), lambda: infer(x=x.data_ptr() + 4), lambda: infer(ids=None), lambda: infer(pred=None),
                 lambda: infer(per_row=0), lambda: train(h=net.h), lambda: train(x=None), lambda: train(ids=None),
                 lambda: train(idx=None), lambda: train(t=None), lambda: train(top=-1), lambda: train(top=1025),
                 lambda: train(y=None), lambda: train(temperature=0.0), lambda: train(alpha=2.0), lambda: train(per_row=-1)):
        assert call() == pnn.PNN_EINVAL
    assert infer(n=-1) == pnn.PNN_ESHAPE and train(n=-1) == pnn.PNN_ESHAPE
    assert L.pnn_last_error(soft.h)
    assert infer(n=0, x=None, ids=None, pred=None) == pnn.PNN_OK and train(n=0, x=None, ids=None) == pnn.PNN_OK
    many = pnn.PNN(pnn.make_config((8, 2), (pnn.SOFTMAX,), pnn.LOSS_XENT, replicas=1025), np.zeros(18, np.float32))
    assert infer(h=many.h) == pnn.PNN_EINVAL and "1..1024" in L.pnn_last_error(many.h).decode()
    with pytest.raises(ValueError):
        net.infer_routed(x, ids, pred[:4])
    infer_pred = torch.empty_like(pred)
    net.infer_routed(x, ids, infer_pred)  # the handles still work
    soft.train_routed(x, ids, idx, t, y, 2.0, 0.5)
    torch.cuda.synchronize()


@gpu
def test_a_deferred_broadcast_is_not_recorded():
    """The copy that a merge leaves to the next call is made by an eager call, not by every replay of a graph."""
    net = network((784, 256, 10), (pnn.SIGMOID, pnn.SOFTMAX), 4, batch=128, lr=0.1)
    assert net.plan == "mini-batch fused last layer"
    x, ids, idx, t, y = (v.cuda() for v in batch(40, 1, net, 5))
    pred = torch.empty(40, dtype=torch.int32, device="cuda")
    net.infer_routed(x, ids, pred)
    net.merge(broadcast=True)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(pnn.PnnError) as e:
        with torch.cuda.graph(graph):
            net.infer_routed(x, ids, pred)
    assert e.value.status == pnn.PNN_EHIP and "broadcast" in str(e.value)
    out = torch.empty(40, 10, device="cuda")
    net.infer_routed(x, ids, pred, out=out)  # makes it
    assert all(np.array_equal(net.get_params(k), net.get_params(-1)) for k in range(4))
    graph = torch.cuda.CUDAGraph()
    kept = torch.empty_like(out)
    with torch.cuda.graph(graph):
        net.infer_routed(x, ids, pred, out=kept)
    for _ in range(3):
        kept.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(kept, out)
