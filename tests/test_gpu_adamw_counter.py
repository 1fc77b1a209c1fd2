"""The counter of steps, which every thread block reads and the last one advances: the same step in all of them, whatever their number."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("sizes", [[1], [2048] * 7, [3_000_000], [700] * 500])
def test_every_block_takes_the_same_step(sizes, bits):
    """With constant gradients of one size a step moves all parameters alike, by as much as its number says; 60 steps, one behind the other."""
    from paper_2608_16305_b200 import destinations as D
    params = [torch.zeros(n, device="cuda") for n in sizes]
    grads = [torch.full((n,), 0.5, device="cuda") for n in sizes]
    grads2 = [torch.zeros(n, device="cuda") for n in sizes]
    opt = D.AdamW(params, lr=0.25, betas=(0.5, 0.75), bits=bits)
    seen = []
    for t in range(60):
        opt.step(grads if t % 3 == 0 else grads2)
        if bits == 32:
            seen.append([(p.min(), p.max()) for p in params])
    assert opt.steps.tolist() == [60, 0]
    for s in seen:
        assert len({float(v) for pair in s for v in pair}) == 1
    m, v = opt.moments()
    if bits == 32:
        assert all(len(torch.unique(x)) == 1 for x in m + v)


def test_a_counter_at_an_odd_place():
    """8-byte alignment is all that is asked of it."""
    from paper_2608_16305_b200 import destinations as D
    out = []
    for at in (0, 1, 3):
        p = torch.ones(100_000, device="cuda")
        opt = D.AdamW([p], bits=8)
        opt.steps = torch.zeros(8, dtype=torch.int64, device="cuda")[at:at + 2]
        for _ in range(5):
            opt.step([torch.full((100_000,), 0.1, device="cuda")])
        assert opt.steps.tolist() == [5, 0]
        out.append(p)
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])
