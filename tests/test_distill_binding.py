"""Teachers that come in halves are refused, on the host."""
import pytest
import torch

from paper_2304_09590_amd import pnn

Z, IDX, T = torch.zeros(4, 10), torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3)


@pytest.mark.parametrize("idx,t,why", [(IDX, None, "together"), (None, T, "together"), (IDX, T[:, :2], "t is"), (IDX[:3], T, "idx is"),
                                       (IDX[0], T[0], "idx is")])
def test_half_a_teacher_is_refused(idx, t, why):
    """Classes without logits, logits without classes (the loss would be 0), and sizes that differ."""
    with pytest.raises(ValueError, match=why):
        pnn.distill_loss(Z, idx, t)
    with pytest.raises(ValueError, match=why):
        pnn.distill_grad(Z, idx, t, torch.zeros(16))
