"""Plans of the AdamW step: their size, and steps that ask for other states or gradients than a plan holds."""
import ctypes

import pytest
import torch

from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu
FAKE = 1 << 20
HEAD, CHUNK = 32 * 64, 72  # places in which workgroups are counted; seven addresses and four words a chunk


@pytest.mark.parametrize("sizes", [(1,), (4096,), (4097, 1), (0, 5, 100000), (0,), (3,) * 100])
def test_a_plan_has_room_for_its_places_and_chunks(sizes):
    chunks = sum(-(-n // 4096) for n in sizes)
    tensors = (pnn.PnnAdamwTensor * len(sizes))(*(pnn.PnnAdamwTensor(FAKE, FAKE, FAKE, FAKE, None, None, None, n) for n in sizes))
    size, count = ctypes.c_int64(), ctypes.c_int64()
    assert pnn.lib().pnn_adamw_bytes(tensors, len(sizes), ctypes.byref(size), ctypes.byref(count)) == pnn.PNN_OK
    assert (size.value, count.value) == (HEAD + CHUNK * chunks, chunks)
    if chunks:  # a byte less is refused
        assert pnn.lib().pnn_adamw_plan(tensors, len(sizes), 32, pnn.FP32, FAKE, size.value - 1, None) == pnn.PNN_ESHAPE


@gpu
@pytest.mark.parametrize("held,asked", [(a, b) for a in ((32, 0), (32, 1), (8, 0), (8, 1)) for b in ((32, 0), (32, 1), (8, 0), (8, 1)) if a != b])
@pytest.mark.parametrize("n", [300, 300_000])
def test_a_step_of_another_kind_than_the_plans_does_nothing(held, asked, n):
    """(Every tensor has room for the widest of its kinds.)"""
    types = (torch.float32, torch.bfloat16)
    assert (pnn.FP32, pnn.BF16_MIXED) == (0, 1)
    memory = [torch.randint(0, 100, (4 * n,), dtype=torch.uint8, device="cuda") for _ in range(4)]
    copy, scales = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), [torch.ones(n, device="cuda") for _ in range(2)]
    dtype = torch.float32 if held[0] == 32 else torch.uint8
    p, g = memory[0].view(torch.float32)[:n], memory[1].view(types[held[1]])[:n]
    state = [[m.view(dtype)[:n]] for m in memory[2:]]
    if held[0] == 8:
        state += [[s[:-(-n // 256)]] for s in scales]
    opt = pnn.AdamW([p], [g], copies=[copy], bits=held[0], state=state)
    all_of = [*memory, copy, *scales, opt.steps, opt._plan]
    before = [t.clone() for t in all_of]
    opt.args.bits, opt.args.g_type = asked
    opt.step()
    assert all(torch.equal(a, b) for a, b in zip(all_of, before))
    opt.args.bits, opt.args.g_type = held
    opt.step()
    assert opt.steps.tolist() == [1, 0] and not torch.equal(memory[0], before[0])


def test_memory_is_the_objects(monkeypatch):
    """A parameter whose data is replaced: the memory that steps write stays the object's."""
    monkeypatch.setattr(pnn, "_on", lambda stream, body, *a, **kw: (torch.zeros(1), 0, 0))
    p, g = torch.zeros(1000), torch.zeros(1000, dtype=torch.bfloat16)
    at = [p.data_ptr(), g.data_ptr()]
    opt = pnn.AdamW([p], [g], copies=[None])
    p.data, g.data = torch.ones(1000), torch.ones(1000, dtype=torch.bfloat16)
    assert set(at) <= {m.data_ptr() for m in opt._memory}
    assert all(t.data_ptr() in {m.data_ptr() for m in opt._memory} for s in opt.state for t in s)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_after_a_parameters_data_was_replaced(bits):
    n = 3_000_000
    p, g = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    opt = pnn.AdamW([p], [g], bits=bits)
    at = p.data_ptr(), g.data_ptr()
    p.data, g.data = torch.full((n,), 5.0, device="cuda"), torch.full((n,), 6.0, device="cuda")
    others = [torch.full((n,), 7.0, device="cuda") for _ in range(4)]
    assert not {t.data_ptr() for t in others} & set(at)
    opt.step()
    assert all((t == 7).all() for t in others) and (p == 5).all() and (g == 6).all() and opt.steps.tolist() == [1, 0]
