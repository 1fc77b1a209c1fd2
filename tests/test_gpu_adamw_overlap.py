"""Tensors that share memory: an AdamW step would write each place twice, in any order."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_tensors_that_overlap_are_refused():
    from paper_2608_16305_b200 import destinations as D
    x, y = torch.zeros(40, device="cuda"), torch.zeros(8, device="cuda")
    half = torch.zeros(40, dtype=torch.bfloat16, device="cuda")
    for params, copies in (([x, x], None), ([x, y, x[39:]], None), ([y, x[:10], x[9:]], None), ([x.view(5, 8), x], None), ([x, y], [half, half[:8]]),
                           ([x, torch.zeros(8, device="cuda")], [half, half[32:]]), ([x], [x.view(torch.bfloat16)[:40]])):
        with pytest.raises(ValueError, match="overlap"):
            D.AdamW(params, copies=copies)
    none = torch.zeros(0, device="cuda")
    D.AdamW([x[:10], x[10:], none, none, x[3:3], y], copies=[half[:10], half[10:], None, None, None, None])
