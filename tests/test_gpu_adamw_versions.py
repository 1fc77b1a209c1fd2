"""Autograd notices that a step has written parameters and their copies."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
def test_a_graph_from_before_the_step_is_refused(bits):
    from paper_2608_16305_b200 import destinations as D
    g = torch.Generator(device="cuda").manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    weights, still = r(40, 16), r(5).requires_grad_()
    table = weights.bfloat16().requires_grad_()
    bias = r(40).requires_grad_()
    opt = D.AdamW([weights, bias.detach(), still], bits=bits, copies=[table.detach(), None, None])
    target = torch.arange(8, dtype=torch.int32, device="cuda")
    loss = D.destination_loss(r(8, 16).bfloat16(), table, target, bias=bias).sum()
    other, third = (bias * bias).sum(), (still * still).sum()
    before = [x._version for x in (weights, table, bias, still)]
    opt.step([torch.ones_like(table), torch.ones_like(bias), None])
    assert [x._version > v for x, v in zip((weights, table, bias, still), before)] == [True, True, True, False]
    for out in (loss, other):
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.backward()
    third.backward()                                     # what had no gradient stayed as it was
    assert torch.equal(still.grad, 2 * still.detach())


def test_tensors_of_inference_mode_are_stepped():
    from paper_2608_16305_b200 import destinations as D
    with torch.inference_mode():
        p = torch.ones(7, device="cuda")
        D.AdamW([p], lr=0.5).step([torch.ones(7, device="cuda")])
    assert float((p - 0.5).abs().max()) < 1e-6
