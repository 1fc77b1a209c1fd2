"""What the destination loss keeps for a backward pass, by grad mode and leaves; the library's call is replaced, so no device is needed."""
import pytest
import torch

from paper_2608_16305_b200 import binding as B
from paper_2608_16305_b200 import destinations as D


@pytest.fixture
def calls(monkeypatch):
    from paper_2608_16305_b200 import build
    build.build_library()
    seen = []
    monkeypatch.setattr(B, "destination_loss", lambda q, table, target, loss, scratch, status, bias=None, kept=None, scale=None:
                        seen.append(kept) or loss.zero_())
    return seen


def args(q_grad, table_grad, bias_grad):
    return (torch.zeros(4, 8, requires_grad=q_grad), torch.zeros(6, 8, requires_grad=table_grad), torch.zeros(4, dtype=torch.int32)), \
        dict(bias=torch.zeros(6, requires_grad=bias_grad))


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_nothing_is_kept_where_no_backward_pass_can_follow(calls, mode):
    for leaves in ((True, True, True), (False, True, False), (False, False, False)):
        a, kw = args(*leaves)
        with mode():
            assert not D.destination_loss(*a, **kw).requires_grad
    a, kw = args(False, False, False)
    D.destination_loss(*a, **kw)
    assert calls == [None] * 4


@pytest.mark.parametrize("leaves", [(True, False, False), (False, True, False), (False, False, True), (True, True, True)])
def test_what_a_backward_pass_needs_is_kept(calls, leaves):
    a, kw = args(*leaves)
    assert D.destination_loss(*a, **kw).requires_grad
    with torch.no_grad(), torch.enable_grad():
        assert D.destination_loss(*a, **kw).requires_grad
    assert [k.numel() for k in calls] == [B.destination_loss_kept(4, 8)] * 2
