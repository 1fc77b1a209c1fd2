"""Decay rates next to 1 in the AdamW step."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("b1,b2", [(0.9, 0.999), (0.9, 0.9999), (0.95, 0.99999), (0.999, 0.999999), (0.0, 0.0)])
def test_the_first_step_is_that_of_the_gradients_sign(b1, b2, bits):
    """At t = 1 the corrections take (1 - beta) out of the moments, whatever the betas: lr * g / (|g| + eps)."""
    from paper_2608_16305_b200 import destinations as D
    g = torch.randn(5000, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    p = torch.zeros(5000, device="cuda")
    D.AdamW([p], lr=0.5, betas=(b1, b2), eps=1e-8, bits=bits).step([g])
    want = -0.5 * g.double() / (g.double().abs() + 1e-8)
    # half steps of 2^-24: 1 - beta is exact; m and v 1 and 2 (of the root 1), the root 1, the corrections 2, product and sum 2, the quotient 4, the product
    # with m and that with lr 2: below 14
    assert float((p.double() - want).abs().max()) <= 0.5 * 14 * 2.0 ** -24


@pytest.mark.parametrize("b1,b2", [(0.9, 0.9999), (0.999, 0.99999)])
def test_constant_gradients_give_the_same_step_for_ever(b1, b2):
    """Both corrected moments of a constant gradient are its own, at any t: what 1 - beta and beta^t are made of is one number."""
    from paper_2608_16305_b200 import destinations as D
    g = torch.full((300,), 0.75, device="cuda")
    p = torch.zeros(300, device="cuda")
    opt = D.AdamW([p], lr=0.5, betas=(b1, b2), eps=0.0)
    for t in range(1, 41):
        before = p.clone()
        opt.step([g])
        # besides the roundings above, those of t steps in the moments (3 half steps of each sum at most), and the parameter's own
        assert float(((before - p).double() - 0.5).abs().max()) <= 0.5 * (14 + 5 * t) * 2.0 ** -24 + float(p.abs().max()) * 2.0 ** -23, t
