"""slot_attention under autograd where part of its inputs takes no part: no bias, leaves without a gradient."""
import numpy as np
import pytest
import torch

from oracle import history as oh

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,KV", [(4, 2), (2, 2), (6, 2)])
@pytest.mark.parametrize("leaves", ["k", "q", "v", "qkv"])
def test_gradients_without_a_bias(heads, KV, leaves):
    from paper_2608_16305_b200 import history as H
    R, S, D = 24, 7, 16
    g = torch.Generator(device="cuda").manual_seed(11)
    mk = lambda *s: torch.randn(*s, generator=g, device="cuda")
    t = {"q": mk(R, heads, D), "k": mk(R, S, KV, D), "v": mk(R, S, KV, D)}
    for x in leaves:
        t[x].requires_grad_()
    cnt = torch.randint(0, S + 1, (R,), generator=g, device="cuda", dtype=torch.int32)
    w = mk(R, heads, D)
    out = H.slot_attention(t["q"], t["k"], t["v"], cnt)
    got = dict(zip(leaves, torch.autograd.grad((out * w).sum(), [t[x] for x in leaves])))
    d = lambda x: x.detach().double().cpu().numpy()
    c = cnt.cpu().numpy()
    args = (d(t["q"]), d(t["k"]), d(t["v"]), c, None, None, D ** -0.5)
    ref = oh.slot_attend(*args)
    # fp32 sums of under a hundred terms
    assert np.abs(d(out) - ref).max() <= 2.0 ** -17 * max(1.0, np.abs(ref).max())
    grads = dict(zip("qkv", oh.slot_attend_backward(*args, d(w))[:3]))
    for x in leaves:
        assert np.abs(grads[x]).max() > 0.1
        assert np.abs(d(got[x]) - grads[x]).max() <= 2.0 ** -17 * max(1.0, np.abs(grads[x]).max()), x
