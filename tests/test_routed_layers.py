"""Routing, grouped products, combining and the optimiser together, as a program trains networks that it routes rows to and
serves them: every gradient against 64-bit differentiation, the handle's calls with a router's ids and gates."""
import numpy as np
import pytest
import torch

import pnn_inputs as I
from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


class Layers:
    """A router and K networks of inputs-hidden-outputs, rectifier between."""

    def __init__(self, K, k, inputs, hidden, outputs, dtype, seed=0):
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, scale=1.0):
            return (torch.randn(*shape, generator=g) * scale).cuda()

        self.K, self.k, self.dtype = K, k, dtype
        self.router = normal(1, K, inputs, scale=inputs ** -0.5)
        self.params = [normal(K, hidden, inputs, scale=inputs ** -0.5), normal(K, hidden, scale=0.1),
                       normal(K, outputs, hidden, scale=hidden ** -0.5), normal(K, outputs, scale=0.1)]
        self.copies = [p.to(BF16) if dtype == BF16 and i % 2 == 0 else None for i, p in enumerate(self.params)]
        if dtype == F32:
            self.copies = [None] * 4
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.router_grad = torch.zeros_like(self.router)

    def weights(self):
        return [c if c is not None else p for c, p in zip(self.copies, self.params)]

    def step(self, x, target, share=0.05, stream=None):
        """Loss gradients of 1/2 sum (out - target)^2 / n + share * balance; the layers' gradients are filled."""
        n, kw = x.shape[0], dict(stream=stream)
        w1, b1, w2, b2 = self.weights()
        one = pnn.group_rows(torch.zeros(n, dtype=torch.int32, device="cuda"), 1, **kw)  # the router is a network of its own
        s = pnn.grouped_forward(one, x.float(), self.router, **kw)
        ids, gates, counts, balance = pnn.route(s, self.k, normalize=True, **kw)
        groups = pnn.group_rows(ids, self.K, **kw)
        pairs = pnn.RowGroups(groups.plan, n * self.k, 1, self.K, groups.stream)
        h = pnn.grouped_forward(groups, x, w1, b1, act=pnn.RELU, **kw)
        y = pnn.grouped_forward(pairs, h, w2, b2, **kw)
        out = pnn.combine_rows(y, ids, gates, self.K, out_dtype=F32, **kw)
        dout = (out - target) / n
        dy, dgates = pnn.combine_grad(dout, y, ids, gates, self.K, **kw)
        pnn.grouped_backward_weights(pairs, dy, h, dw=self.grads[2], db=self.grads[3], **kw)
        dh = pnn.grouped_backward_input(pairs, dy, w2, a=h, act=pnn.RELU, **kw)
        pnn.grouped_backward_weights(groups, dh, x, dw=self.grads[0], db=self.grads[1], **kw)
        dl = torch.full((1,), share, device="cuda")
        ds = pnn.route_grad(s, ids, counts, dgates, dl, normalize=True, **kw)
        pnn.grouped_backward_weights(one, ds, x.float(), dw=self.router_grad, bias=False, **kw)
        return ids, gates, counts, balance, out

    def reference(self, x, target, ids, share=0.05):
        """The same in 64 bits by automatic differentiation, the choice of networks given."""
        x = x.double().cpu()
        params = [p.double().cpu().requires_grad_(True) for p in self.weights()]
        router = self.router.double().cpu().requires_grad_(True)
        w1, b1, w2, b2 = params
        n, at = x.shape[0], ids.long().cpu()
        s = x @ router[0].T
        p = torch.softmax(s, 1)
        gates = torch.softmax(s.gather(1, at), 1)
        counts = torch.bincount(at.flatten(), minlength=self.K).double()
        balance = self.K * (counts / counts.sum() * p.sum(0)).sum() / n
        out = 0
        for j in range(self.k):
            h = torch.relu((w1[at[:, j]] @ x[:, :, None])[:, :, 0] + b1[at[:, j]])
            out = out + gates[:, j:j + 1] * ((w2[at[:, j]] @ h[:, :, None])[:, :, 0] + b2[at[:, j]])
        loss = 0.5 * ((out - target.double().cpu()) ** 2).sum() / n + share * balance
        return balance.item(), out.detach(), [g.detach() for g in torch.autograd.grad(loss, params + [router])]


def off(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


@gpu
@pytest.mark.parametrize("dtype,bar", [(F32, 2e-5), (BF16, 3e-2)])
@pytest.mark.parametrize("n,K,k,inputs,hidden,outputs", [(1, 3, 2, 16, 8, 4), (50, 5, 1, 24, 40, 10), (300, 12, 3, 37, 29, 11), (2000, 40, 2, 64, 128, 16)])
def test_gradients_of_a_routed_step(n, K, k, inputs, hidden, outputs, dtype, bar):
    """Normwise: fp32 sums of some hundred terms are off by 1e-6 of their terms; bf16 rows, weights, activations and
    errors by 2^-8 each, in four products after each other."""
    net = Layers(K, k, inputs, hidden, outputs, dtype)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(n, inputs, generator=g).to(dtype).cuda()
    target = torch.randn(n, outputs, generator=g).cuda()
    ids, gates, counts, balance, out = net.step(x, target)
    value, want, grads = net.reference(x, target, ids)
    assert abs(float(balance) - value) <= 1e-5 * value and int(counts[-1]) == n
    assert off(out, want) <= bar
    for got, w in zip(net.grads, grads[:4]):
        assert off(got, w) <= bar
    # (router: the gates' and the balance loss's gradient through the scores)
    assert off(net.router_grad, grads[4]) <= 2 * bar


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_recorded_steps_of_training_are_the_eager_ones(dtype, bits):
    """Step and optimiser in one graph, replayed: the same bits as eager steps, which go on in between."""
    x = torch.randn(200, 24, generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    target = torch.randn(200, 10, generator=torch.Generator().manual_seed(3)).cuda()

    def made():
        net = Layers(6, 2, 24, 16, 10, dtype, seed=4)
        return net, pnn.AdamW(net.params + [net.router], net.grads + [net.router_grad], copies=net.copies + [None], bits=bits, lr=1e-2)

    eager, e = made()
    recorded, r = made()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = recorded.step(x, target)
        r.step()
    for _ in range(4):
        graph.replay()
        got = eager.step(x, target)
        e.step()
        torch.cuda.synchronize()
        for a, b in zip(kept, got):
            assert torch.equal(a, b)
        for a, b in zip(r.params + r.grads + sum(r.state, []) + [r.steps], e.params + e.grads + sum(e.state, []) + [e.steps]):
            assert torch.equal(a, b)
        assert all(torch.equal(a, b) for a, b in zip(recorded.copies, eager.copies) if a is not None)
        x.mul_(-0.9)


@gpu
def test_served_from_codes():
    """The same layers from 8-bit codes: off from the fp32 ones by the codes' roundings (half a code of operands whose
    largest is three to four times their root mean square: 1 % a product)."""
    net = Layers(12, 2, 100, 64, 16, F32)
    x = torch.randn(500, 100, generator=torch.Generator().manual_seed(5)).cuda()
    ids, gates, _, _, out = net.step(x, torch.zeros(500, 16, device="cuda"))
    w1, b1, w2, b2 = net.weights()
    groups = pnn.group_rows(ids, 12)
    pairs = pnn.RowGroups(groups.plan, 1000, 1, 12, groups.stream)
    h = pnn.grouped_forward_int8(groups, *pnn.quantize_rows(x), *pnn.quantize_rows(w1), b1, act=pnn.RELU)
    y = pnn.grouped_forward_int8(pairs, *pnn.quantize_rows(h), *pnn.quantize_rows(w2), b2)
    got = pnn.combine_rows(y, ids, gates, 12)
    assert off(got, out.double().cpu()) <= 0.04


@gpu
def test_a_router_in_front_of_the_handles_calls():
    """pnn_infer_routed with a router's ids and gates gives the gates' mean of the single networks' answers."""
    w = I.WORKLOADS[1].scaled(replicas=4)
    cfg = pnn.config_from_workload(w)
    g = np.random.default_rng(7)
    net = pnn.PNN(cfg, I.init_params(w))
    for e in range(4):
        net.set_params(e, (0.1 * g.standard_normal(net.P)).astype(np.float32))
    n, O = 300, cfg.sizes[cfg.n_layers]
    x = torch.from_numpy(g.random((n, cfg.sizes[0]), dtype=np.float32)).cuda()
    s = torch.from_numpy(g.standard_normal((n, 4)).astype(np.float32)).cuda()
    s[5] = -float("inf")  # a row that goes nowhere
    ids, gates, _, _ = pnn.route(s, 2, normalize=True)
    pred, out = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, O, device="cuda")
    net.infer_routed(x, ids, pred, weights=gates, out=out)
    single, answers = torch.empty(n, O, device="cuda"), []
    for e in range(4):
        net.infer(x, torch.empty_like(pred), which=e, out=single)
        answers.append(single.clone())
    answers = torch.stack(answers, 1)
    want = (answers.gather(1, ids.clamp(min=0).long()[:, :, None].expand(n, 2, O)) * gates[:, :, None]).sum(1)
    assert (out - want).abs().max() <= 1e-5 and (out[5] == 0).all() and int(pred[5]) == -1
    net.close()
