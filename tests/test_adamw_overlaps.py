"""Gradients in the memory of what an AdamW step writes: of their own tensor and value by value they are read first, anything else
would be read while others write it."""
import pytest
import torch

from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def test_gradients_in_what_a_step_writes_are_refused():
    a, b, half = torch.zeros(3000), torch.zeros(3000), torch.zeros(3000, dtype=BF16)
    m, v = torch.zeros(1000), torch.zeros(1000)
    steps = torch.zeros(300, dtype=torch.int32)
    for p, g, kw in (
            ([a[:1000]], [a[500:1500]], {}), ([a[:1000]], [a[999:1999]], {}), ([a[500:1500]], [a[:1000]], {}),
            ([a[:1000], a[1000:2000]], [a[1000:2000], b[:1000]], {}),                        # (another tensor's)
            ([a[:1000]], [a.view(BF16)[:1000]], {}), ([a[:1000]], [m.view(BF16)[500:1500]], dict(state=[[m], [v]])),
            ([a[:1000]], [v[1:].view(BF16)[:1000]], dict(state=[[m], [v]])), ([a[:1000]], [half[1:1001]], dict(copies=[half[:1000]])),
            ([a[:1000]], [half[:2000].view(F32)], dict(copies=[half[:1000]])), ([a[:1000]], [b[:1000]], dict(steps=a.view(torch.int32)[998:1000])),
            ([a[:100]], [steps[:100].view(F32)], dict(steps=steps[99:101])), ([a[:1000]], [b[:1000]], dict(lr=a[3:4])),
            ([a[:1000]], [b[:1000]], dict(lr=m[5:6], state=[[m], [v]]))):
        with pytest.raises(ValueError, match="overlap"):
            pnn.AdamW(p, g, **kw)
    # value by value, beside each other, shared by two tensors, empty: only the device is missing
    for p, g, kw in (([a[:1000]], [a[:1000]], {}), ([a[:1000]], [m], dict(state=[[m], [v]])), ([a[:1000]], [half[:1000]], dict(copies=[half[:1000]])),
                     ([a[:1000], a[2000:]], [a[1000:2000], b[:1000]], {}), ([a[:1000], a[1000:2000]], [b[:1000], b[:1000]], {}),
                     ([a[:0], a[:1000]], [a[5:5], b[:1000]], {}), ([a[:1000]], [b[:1000]], dict(lr=b[3:4]))):
        with pytest.raises(ValueError, match="CUDA"):
            pnn.AdamW(p, g, **kw)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [7, 5000, 2_000_003])
def test_gradients_value_by_value_in_the_same_memory(n, bits):
    gen = torch.Generator().manual_seed(n)
    p = torch.randn(n, generator=gen).cuda()
    want = p.clone()
    pnn.AdamW([want], [p.clone()], bits=bits, lr=0.1).step()
    pnn.AdamW([p], [p], bits=bits, lr=0.1).step()
    assert torch.equal(p, want)
    copy = torch.randn(n, generator=gen).to(BF16).cuda()
    q, old = p.clone(), copy.clone()
    pnn.AdamW([want], [old], bits=bits, lr=0.1).step()
    pnn.AdamW([q], [copy], copies=[copy], bits=bits, lr=0.1).step()
    assert torch.equal(q, want) and torch.equal(copy, want.to(BF16))
