"""The smallest eps of the AdamW step, and what is smaller."""
import pytest
import torch

from paper_2608_16305_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
def test_values_without_gradients_stay(bits):
    from paper_2608_16305_b200 import destinations as D
    g = torch.zeros(600, device="cuda")
    g[:100] = 1.0
    for eps in (1e-8, 2.0 ** -126):
        p = torch.full((600,), 3.0, device="cuda")
        D.AdamW([p], eps=eps, lr=0.5, bits=bits).step([g])
        assert bool((p[100:] == 3.0).all()) and float((p[:100] - 2.5).abs().max()) < 1e-5
    for eps in (1e-40, 2.0 ** -127):
        p = torch.full((600,), 3.0, device="cuda")
        opt = D.AdamW([p], eps=eps, lr=0.5, bits=bits)
        with pytest.raises(B.TgnnError, match="eps"):
            opt.step([g])
        assert bool((p == 3.0).all()) and opt.steps.tolist() == [0, 0]
