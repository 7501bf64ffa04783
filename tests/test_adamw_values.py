"""What adamw_values refuses, on the host and with tensors of the GPU."""
import pytest
import torch

from paper_2304_09590_amd import pnn

gpu = pytest.mark.gpu


def parts(n, device):
    return [torch.zeros(n, dtype=torch.uint8, device=device) for _ in range(2)] + [torch.zeros(-(-n // 256), device=device) for _ in range(2)]


def test_tensors_of_the_host_are_refused():
    with pytest.raises(ValueError, match="CUDA"):
        pnn.adamw_values(*parts(300, "cpu"))


@gpu
def test_states_of_other_types_and_sizes_are_refused():
    m, v, ms, vs = parts(300, "cuda")
    for a, why in (((m.float(), v, ms, vs), "m is"), ((m, v.float(), ms, vs), "v is"), ((m, v[:299], ms, vs), "v is"), ((m, v, ms[:1], vs), "m_scale is"),
                   ((m, v, ms, vs.double()), "v_scale is"), ((m, v, ms, torch.zeros(3, device="cuda")), "v_scale is"),
                   ((m.view(20, 15).T, v.view(15, 20), ms, vs), "m is"), ((m, v.cpu(), ms, vs), "tensors on"), ((m, v, ms, vs.cpu()), "tensors on")):
        with pytest.raises(ValueError, match=why):
            pnn.adamw_values(*a)
    got = pnn.adamw_values(m.view(15, 20), v.view(15, 20), ms, vs)
    assert all(x.shape == (15, 20) and (x == 0).all() for x in got)
    assert all(x.shape == (0,) for x in pnn.adamw_values(*parts(0, "cuda")))
