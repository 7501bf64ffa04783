"""Calls of routing, combining, codes and AdamW at the ends of their ranges: the widest and longest, nothing kept, several
threads and streams at once, temporaries of another stream."""
import threading

import pytest
import torch

from paper_2304_09590_amd import pnn
from tests.test_combine import verify as verify_combine
from tests.test_int8 import case as int8_case, codes_of, verify as verify_int8
from tests.test_route import case as route_case, verify as verify_route

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [63, 64, 65, 127, 257, 1025])
@pytest.mark.parametrize("K,k", [(16, 16), (17, 2), (64, 64), (65, 3), (128, 1), (129, 64), (256, 33), (257, 64), (512, 2), (513, 64), (1024, 17)])
def test_routes_about_a_workgroups_rows(n, K, k, dtype):
    s, dgates = route_case(n, K, k, dtype, seed=n + K)
    verify_route(s, k, True, dgates)


@gpu
@pytest.mark.parametrize("K", [10, 100, 300, 1000])
def test_bf16_scores_that_are_no_numbers(K):
    """NaN of both signs and infinities; subnormal scores and both zeros are numbers."""
    s, dgates = route_case(12, K, 3, BF16, seed=1)
    raw = s.view(torch.int16)
    raw[1, 0], raw[2, 1], raw[3, 2] = 0x7FC0, -64, 0x7F81  # (quiet, negative, signalling)
    s[4, 5] = float("inf")
    raw[5] = 1                                             # all at the smallest subnormal
    raw[6] = 0
    raw[6, ::2] = -32768                                   # zeros of both signs: ties
    raw[7, 3:] = -128                                      # three scores, the others -inf
    ids, gates, counts, loss, ds = verify_route(s, 3, False, dgates)
    assert (ids[1:5] == -1).all() and torch.isnan(gates[1:5]).all() and torch.isnan(loss).all()
    assert ids[5].tolist() == ids[6].tolist() == [0, 1, 2] and sorted(ids[7].tolist()) == [0, 1, 2]


@gpu
def test_many_and_wide_pairs():
    for n, k, M in ((3, 1000, 9), (2, 2, 1 << 20), (1, 5, 70000)):
        g = torch.Generator().manual_seed(n)
        y = torch.randn(n * k, M, generator=g).cuda()
        ids = torch.randint(-1, 9, (n, k), generator=g, dtype=torch.int32).cuda()
        verify_combine(y, torch.randn(n, M, generator=g).cuda(), ids, torch.randn(n, k, generator=g).cuda())


@gpu
def test_the_widest_codes():
    x = torch.randn(3, 1 << 20, generator=torch.Generator().manual_seed(2)).cuda()
    q, s = pnn.quantize_rows(x)
    want, scale = codes_of(x)
    assert torch.equal(q.cpu(), want) and torch.equal(s.cpu(), scale)
    # rows apart, and a view that starts inside an allocation
    q, s = pnn.quantize_rows(x[:, 5:1005])
    want, scale = codes_of(x[:, 5:1005])
    assert torch.equal(q.cpu(), want) and torch.equal(s.cpu(), scale)


@gpu
@pytest.mark.parametrize("n,k,K", [(40, 2, 1024), (3000, 1, 1024), (700, 3, 2)])
def test_networks_without_pairs_and_pairs_without_networks(n, k, K):
    ids, x, xs, w, ws, b = int8_case(n, k, K, 32, 24, seed=1)
    ids[ids % 3 == 0] = -7
    verify_int8(ids, x, xs, w, ws, b, "relu", F32, K)
    ids.fill_(K)  # nothing is kept
    xs.fill_(float("nan"))
    _, y = verify_int8(ids, x, xs, w, ws, b, "sigmoid", BF16, K)
    assert (y == 0).all()
    out = pnn.combine_rows(y, ids, torch.full((n, k), float("inf"), device="cuda"), K)
    dy, dw = pnn.combine_grad(out, y, ids, torch.full((n, k), float("nan"), device="cuda"), K)
    assert (out == 0).all() and (dy == 0).all() and (dw == 0).all()


@gpu
def test_several_threads_at_once():
    """Each thread with its own stream, rows and optimiser: the results of the calls made alone."""
    def work(seed, stream):
        with torch.cuda.stream(stream):
            g = torch.Generator(device="cuda").manual_seed(seed)
            s = torch.randn(3000, 40 + seed, generator=g, device="cuda")
            out = []
            p, d = torch.zeros(5000, device="cuda"), torch.randn(5000, generator=g, device="cuda")
            opt = pnn.AdamW([p], [d], bits=8, seed=seed)
            for _ in range(20):
                ids, gates, counts, loss = pnn.route(s, 2)
                ds = pnn.route_grad(s, ids, counts, gates, loss)
                y = torch.randn(6000, 30, generator=g, device="cuda")
                out.append((ids, gates, counts, loss, ds, pnn.combine_rows(y, ids, gates, 40 + seed), *pnn.quantize_rows(ds)))
                opt.step()
                s = s * 0.9 + ds
            stream.synchronize()
        return out + [(p, *sum(opt.state, []), opt.steps)]

    alone = [work(i, torch.cuda.Stream()) for i in range(4)]
    got = [None] * 4

    def one(i, stream):
        got[i] = work(i, stream)

    threads = [threading.Thread(target=one, args=(i, torch.cuda.Stream())) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for a, b in zip(alone, got):
        assert all(torch.equal(x, y) for u, v in zip(a, b) for x, y in zip(u, v))


@gpu
def test_temporaries_of_another_stream_are_kept():
    """A busy stream takes calls with temporaries of the default stream, whose memory is asked for again at once."""
    n, K, side = 50000, 200, torch.cuda.Stream()
    s = torch.randn(n, K, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    want = pnn.route(s * 1, 2)
    grad = pnn.route_grad(s, *want[:1], want[2], want[1], want[3])
    codes = pnn.quantize_rows(s * 2)
    rows = pnn.combine_rows(s[:n], want[0][:n // 2], want[1][:n // 2], K)
    torch.cuda.synchronize()
    busy = torch.randn(4096, 4096, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy * 1e-4
    ts = [s * 1, want[0] * 1, want[2] * 1, want[1] * 1, want[3] * 1, s * 2, s * 1]
    torch.cuda.current_stream().synchronize()
    got = pnn.route(ts[0], 2, stream=side)
    g2 = pnn.route_grad(ts[6], ts[1], ts[2], ts[3], ts[4], stream=side)
    c2 = pnn.quantize_rows(ts[5], stream=side)
    r2 = pnn.combine_rows(ts[6][:n], ts[1][:n // 2], ts[3][:n // 2], K, stream=side)
    del ts
    junk = [torch.full((n, K), 9.0, device="cuda") for _ in range(4)] + [torch.full((n, 2), 9, dtype=torch.int32, device="cuda") for _ in range(4)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(g2, grad) and torch.equal(r2, rows)
    assert all(torch.equal(a, b) for a, b in zip(c2, codes)) and len(junk) == 8


@gpu
def test_steps_of_two_graphs_in_turn():
    """Two optimisers' steps recorded, replayed in turn with eager steps of a third on the same gradients."""
    g = torch.randn(10000, device="cuda")

    def made():
        p = torch.zeros(10000, device="cuda")
        return p, pnn.AdamW([p], [g], bits=8, seed=5)

    (pa, a), (pb, b), (pc, c) = made(), made(), made()
    graphs = []
    for o in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o.step()
            o.step()
        graphs.append(graph)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        c.step()
        c.step()
        torch.cuda.synchronize()
        assert torch.equal(pa, pb) and torch.equal(pa, pc) and a.steps.tolist() == c.steps.tolist()
        g.mul_(-0.5)
