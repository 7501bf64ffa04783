"""Tensors that a call takes to another stream than their own: the binding records them there, so that a
temporary's memory is not given to others while the call's work may still read it."""
import contextlib
import types

import numpy as np
import pytest
import torch

from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu


# ---- what is recorded, on the host: stand-ins for torch's streams and tensors ---------------------

class Stream:
    def __init__(self, handle, device="cuda:0"):
        self.cuda_stream, self.device = handle, device


class External(Stream):
    def __init__(self, handle, device):
        super().__init__(handle, device)


class Tensor:
    is_cuda, device = True, "cuda:0"

    def __init__(self, shape=(4, 8), dtype="torch.float32"):
        self.shape, self.dtype, self.on = shape, dtype, []

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def record_stream(self, stream):
        self.on.append(stream)


@pytest.fixture
def fake(monkeypatch):
    """torch as the binding sees it: device 0 and a current stream of handle 7."""
    cuda = types.SimpleNamespace(Stream=Stream, ExternalStream=External, device=lambda d: contextlib.nullcontext(),
                                 stream=lambda s: contextlib.nullcontext(), current_stream=lambda d=None: current)
    current = Stream(7)
    c = types.SimpleNamespace(_cuda_getDevice=lambda: 0, _cuda_getCurrentRawStream=lambda d: current.cuda_stream)
    monkeypatch.setattr(pnn, "_torch", types.SimpleNamespace(cuda=cuda, _C=c))
    return current


def test_tensors_are_recorded_on_a_given_stream(fake):
    side, a, b = Stream(9), Tensor(), Tensor()
    groups = types.SimpleNamespace(plan=Tensor(), stream=7)
    assert pnn._on(side, lambda s: s, a, None, b, groups=groups) == 9
    assert a.on == b.on == groups.plan.on == [side]
    # a raw handle is the caller's; the current stream is torch's own rule
    for stream, handle in ((11, 11), (None, 7)):
        x, plan = Tensor(), types.SimpleNamespace(plan=Tensor(), stream=7)
        assert pnn._on(stream, lambda s: s, x, groups=plan) == handle
        assert x.on == plan.plan.on == []


def test_a_plan_of_another_stream_is_recorded_on_the_current_one(fake):
    for made_on in (9, None):
        groups = types.SimpleNamespace(plan=Tensor(), stream=made_on)
        pnn._on(None, lambda s: s, Tensor(), groups=groups)
        assert groups.plan.on == [fake]


@pytest.mark.parametrize("call,given", [
    ("pnn_train_epoch", lambda n, t, s: n.train_epoch(t["x"], t["y"], stream=s)),
    ("pnn_train_epoch_order", lambda n, t, s: n.train_epoch_order(t["x"], t["y"], t["pred"], stream=s)),
    ("pnn_infer", lambda n, t, s: n.infer(t["x"], t["pred"], out=t["out"], y=t["y"], stream=s)),
    ("pnn_eval", lambda n, t, s: n.evaluate(t["x"], t["y"], stream=s)),
    ("pnn_eval_noalloc", lambda n, t, s: n.evaluate_noalloc(t["x"], t["y"], stream=s)),
    ("pnn_infer_routed", lambda n, t, s: n.infer_routed(t["x"], t["ids"], t["pred"], t["weights"], t["out"], stream=s)),
    ("pnn_train_routed", lambda n, t, s: n.train_routed(t["x"], t["ids"], t["idx"], t["t"], t["y"], 1.0, 0.5, t["weights"], stream=s))])
def test_the_handles_calls_record(fake, call, given):
    i32 = "torch.int32"
    tensors = {"x": Tensor(), "y": Tensor((4,), i32), "pred": Tensor((4,), i32), "out": Tensor((4, 3)), "ids": Tensor((4, 2), i32),
               "weights": Tensor((4, 2)), "idx": Tensor((4, 2), i32), "t": Tensor((4, 2))}
    net = object.__new__(pnn.PNN)
    net.h, net.cfg = None, pnn.make_config((8, 3), (pnn.SOFTMAX,), pnn.LOSS_XENT)
    passed = []
    net._lib = types.SimpleNamespace(**{call: lambda *a: passed.append(a) or pnn.PNN_OK})
    used = {"pnn_train_epoch": "x y", "pnn_train_epoch_order": "x y pred", "pnn_infer": "x pred out y", "pnn_eval": "x y",
            "pnn_eval_noalloc": "x y", "pnn_infer_routed": "x ids pred weights out", "pnn_train_routed": "x ids idx t y weights"}[call]
    side = Stream(9)
    given(net, tensors, side)
    assert passed[0][-1] == 9
    assert {k for k, t in tensors.items() if t.on == [side]} == set(used.split())
    for t in tensors.values():
        t.on = []
    for stream, handle in ((11, 11), (None, 7)):
        given(net, tensors, stream)
        assert passed[-1][-1] == handle and not any(t.on for t in tensors.values())


# ---- on the GPU ------------------------------------------------------------------------------------

def reused(t):
    """Whether the memory of a tensor that goes away is given to the next one of its size."""
    at, shape, dtype = t.data_ptr(), t.shape, t.dtype

    def after():
        return torch.empty(shape, dtype=dtype, device="cuda").data_ptr() == at

    return after


@gpu
def test_memory_of_temporaries_is_kept_until_the_work_has_ended():
    """A stream that is busy for a while, calls on it with temporaries of the default stream, new tensors at once."""
    n, side = 300000, torch.cuda.Stream()
    ids = torch.randint(0, 5, (n, 2), dtype=torch.int32)
    x = torch.randn(n, 8)
    w = torch.randn(5, 16, 8, device="cuda")
    want = pnn.grouped_forward(pnn.group_rows(ids.cuda(), 5), x.cuda(), w)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    ids_dev, x_dev = ids.cuda(), x.cuda()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    ended = torch.cuda.Event()
    groups = pnn.group_rows(ids_dev, 5, stream=side)
    got = pnn.grouped_forward(groups, x_dev, w, stream=side)
    ended.record(side)
    again = [reused(ids_dev), reused(x_dev)]
    del ids_dev, x_dev
    taken = [f() for f in again]
    busy = not ended.query()
    side.synchronize()
    assert torch.equal(got, want)
    assert busy and not any(taken)


@gpu
def test_memory_of_a_plan_is_kept_until_another_streams_work_has_ended():
    n, side = 300000, torch.cuda.Stream()
    ids, x = torch.randint(0, 5, (n, 2), dtype=torch.int32, device="cuda"), torch.randn(n, 8, device="cuda")
    w = torch.randn(5, 16, 8, device="cuda")
    want = pnn.grouped_forward(pnn.group_rows(ids, 5), x, w)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    groups = pnn.group_rows(ids, 5, stream=side)
    side.synchronize()
    ended = torch.cuda.Event()
    torch.cuda._sleep(200_000_000)
    got = pnn.grouped_forward(groups, x, w)
    ended.record()
    again = reused(groups.plan)
    del groups
    with torch.cuda.stream(side):
        taken = again()
    busy = not ended.query()
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    assert busy and not taken


@gpu
def test_a_plan_made_outside_a_graph():
    n, networks = 700, 3
    ids = torch.randint(0, networks, (n, 2), dtype=torch.int32, device="cuda")
    x, w = torch.randn(n, 40, device="cuda"), torch.randn(networks, 24, 40, device="cuda")
    groups = pnn.group_rows(ids, networks)
    pnn.grouped_forward(groups, x, w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = pnn.grouped_forward(groups, x, w)
    for _ in range(3):
        x.mul_(-0.5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, pnn.grouped_forward(groups, x, w))


@gpu
def test_the_handles_calls_on_another_stream():
    cfg = pnn.make_config((64, 10), (pnn.SOFTMAX,), pnn.LOSS_XENT, replicas=3)
    net = pnn.PNN(cfg, np.random.default_rng(1).uniform(-1, 1, pnn.param_count(cfg)).astype(np.float32))
    n, side = 100000, torch.cuda.Stream()
    ids, x = torch.randint(0, 3, (n, 1), dtype=torch.int32), torch.rand(n, 64)
    pred, want = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
    net.infer_routed(x.cuda(), ids.cuda(), want)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    ids_dev, x_dev = ids.cuda(), x.cuda()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    net.infer_routed(x_dev, ids_dev, pred, stream=side)
    ended = torch.cuda.Event()
    ended.record(side)
    again = [reused(ids_dev), reused(x_dev)]
    del ids_dev, x_dev
    taken = [f() for f in again]
    busy = not ended.query()
    side.synchronize()
    assert torch.equal(pred, want)
    assert busy and not any(taken)
