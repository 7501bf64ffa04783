"""An AdamW object stepped on another stream than it was made on: its plan, its step count and its states are recorded there, so
that their memory is not given to others while a step that still waits may use it."""
import contextlib
import types

import pytest
import torch

from paper_2304_09590_amd import pnn
from tests.test_binding_streams import External, Stream, Tensor as StandIn, reused

gpu = pytest.mark.gpu


# ---- what is recorded, on the host ------------------------------------------------------------------

class Tensor(StandIn):
    made = 0

    def __init__(self, shape, dtype):
        super().__init__(tuple(shape), dtype)
        Tensor.made += 1
        self.at = Tensor.made << 20

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def data_ptr(self):
        return self.at

    def untyped_storage(self):
        return self

    def new_empty(self, shape, dtype=None):
        return Tensor((shape,) if isinstance(shape, int) else shape, dtype or self.dtype)


@pytest.fixture
def fake(monkeypatch):
    """torch as the binding sees it, device 0; `.handle` is the current stream's; calls of the library end well."""
    now = Stream(7)

    def zeros(*shape, dtype=torch.float32, device=None):
        return Tensor(shape[0] if isinstance(shape[0], tuple) else shape, dtype)

    cuda = types.SimpleNamespace(Stream=Stream, ExternalStream=External, device=lambda d: contextlib.nullcontext(),
                                 stream=lambda s: contextlib.nullcontext(), current_stream=lambda d=None: Stream(now.cuda_stream))
    c = types.SimpleNamespace(_cuda_getDevice=lambda: 0, _cuda_getCurrentRawStream=lambda d: now.cuda_stream)
    monkeypatch.setattr(pnn, "_torch", types.SimpleNamespace(cuda=cuda, _C=c, zeros=zeros, is_tensor=lambda x: isinstance(x, Tensor),
                                                             float32=torch.float32, bfloat16=torch.bfloat16, uint8=torch.uint8, int32=torch.int32))
    now.calls = []
    monkeypatch.setattr(pnn, "_call", lambda what, *a: now.calls.append((what, a[-1])))
    return now


def made(bits, lr=1e-3, **kw):
    params, grads = [Tensor((300,), torch.float32), Tensor((2, 5), torch.float32)], [Tensor((300,), torch.bfloat16), Tensor((2, 5), torch.bfloat16)]
    return pnn.AdamW(params, grads, copies=[Tensor((300,), torch.bfloat16), None], bits=bits, lr=lr, **kw)


def own(opt):
    return [opt._plan, opt.steps, *(t for s in opt.state for t in s)]


def handles(t):
    return {s.cuda_stream for s in t.on}


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_under_another_current_stream_records(fake, bits):
    opt = made(bits)
    opt.step()
    assert not any(t.on for t in own(opt))  # (where it was made: its memory's own stream)
    for handle in (9, 11, 9):
        fake.cuda_stream = handle
        opt.step()
        assert fake.calls[-1] == ("pnn_adamw_step", handle)
    assert all(handles(t) == {9, 11} for t in own(opt))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_on_a_given_stream_records(fake, bits):
    rate = Tensor((1,), torch.float32)
    opt = made(bits, rate)
    opt.step(stream=Stream(9))
    assert fake.calls[-1] == ("pnn_adamw_step", 9)
    used = own(opt) + opt.params + opt.grads + opt.copies[:1] + [rate]
    assert all(handles(t) == {9} for t in used)
    opt.step(stream=13)  # (a raw handle is the caller's)
    assert fake.calls[-1] == ("pnn_adamw_step", 13) and all(handles(t) == {9} for t in used)


def test_states_and_steps_that_are_given_belong_to_the_object(fake):
    state = [[Tensor((300,), torch.float32), Tensor((2, 5), torch.float32)] for _ in "mv"]
    opt = made(32, state=state, steps=Tensor((2,), torch.int32))
    fake.cuda_stream = 9
    opt.step()
    assert all(handles(t) == {9} for t in own(opt))


# ---- on the GPU ---------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
def test_memory_of_an_object_that_goes_away_is_kept(bits, given):
    """Made on the default stream, stepped on a busy one, dropped at once: nobody gets its memory before the step has ended."""
    n, side = 5_000_000, torch.cuda.Stream()
    g = torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    want = torch.zeros(n, device="cuda")
    pnn.AdamW([want], [g], bits=bits, seed=3).step()
    p = torch.zeros(n, device="cuda")
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    opt = pnn.AdamW([p], [g], bits=bits, seed=3)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        if not given:
            opt.step()
    if given:
        opt.step(stream=side)
    ended = torch.cuda.Event()
    ended.record(side)
    again = [reused(t) for t in (opt._plan, opt.state[0][0], opt.state[1][0])]
    del opt
    taken = [f() for f in again]
    busy = not ended.query()
    side.synchronize()
    assert torch.equal(p, want)
    assert busy and not any(taken)
