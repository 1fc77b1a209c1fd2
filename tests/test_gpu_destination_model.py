"""Lookup, attention over sampled slots, destination loss and AdamW together, as a training step uses them."""
import numpy as np
import pytest
import torch

from paper_2608_16305_b200 import workload as wl

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def stream():
    return wl.make_stream(wl.scaled(wl.CONFIGS["tiny"], num_nodes=150, num_events=2000, batch=90))


@pytest.fixture(scope="module")
def workload(stream):
    from paper_2608_16305_b200.trainer import DeviceWorkload
    return DeviceWorkload(stream)


def reference(model, nodes, times, destinations):
    """The losses in 64 bits and their leaves, over the slots that the model samples."""
    table, bias, age = (x.detach().double().clone().requires_grad_() for x in model.leaves)
    s = model.slots(nodes, times)
    own = table[nodes.long()]
    shape = (model.heads, model.dim)
    rows = table[s.nbr.long().clamp(min=0)].view(*s.nbr.shape, *shape)
    q = own.view(-1, *shape)
    place = (times[:, None] - s.ts)[..., None] >= model.age.bounds
    z = torch.einsum("nhd,nshd->nhs", q, rows) * model.dim ** -0.5 + age[:, place.sum(-1)].transpose(0, 1)
    hidden = torch.arange(model.window, device=nodes.device)[None] >= s.cnt[:, None]
    z = z.masked_fill(hidden[:, None], -torch.inf)
    some = (s.cnt > 0)[:, None, None]
    a = torch.where(some, torch.softmax(torch.where(some, z, 0.0), -1), 0.0)
    x = own + torch.einsum("nhs,nshd->nhd", a, rows).reshape(own.shape)
    logits = x @ table.T * (model.heads * model.dim) ** -0.5 + bias
    live = destinations >= 0
    loss = torch.where(live, torch.logsumexp(logits, 1) - logits.gather(1, destinations.long().clamp(min=0)[:, None])[:, 0], 0.0)
    return loss, (table, bias, age), x.detach()


@pytest.mark.parametrize("heads,dim,window", [(2, 16, 10), (1, 50, 3), (4, 33, 1)])
def test_loss_and_gradients(workload, heads, dim, window):
    from paper_2608_16305_b200 import destinations as D
    m = D.DestinationModel(workload, heads=heads, dim=dim, window=window, seed=3)
    with torch.no_grad():
        m.bias.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
        m.age.table.normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    nodes, times, dst = m.targets(5)
    dst = dst.clone()
    dst[::7] = -1
    w = torch.linspace(0.5, 1.5, dst.numel(), device="cuda")
    got = m.loss(nodes, times, dst)
    grads = torch.autograd.grad(got, m.leaves, grad_outputs=w)
    ref, leaves, x = reference(m, nodes, times, dst)
    want = torch.autograd.grad((ref * w.double()).sum(), leaves)
    wide, X, T = heads * dim, float(x.abs().max()), float(m.table.detach().abs().max())
    # What a root attends to is off by 2^-17 of its largest value (weights from fp32 sums of fewer than 100 terms), a logit by that times the row's
    # magnitudes over sqrt(wide), and by 2^-20 of its own largest size; a loss by twice a logit.
    logit = (2.0 ** -17 + 2.0 ** -20) * X * T * wide ** 0.5 + 2.0 ** -20
    assert float((got.detach().double() - ref.detach()).abs().max()) <= 2 * logit
    # Every weight of the softmax is off by 2 logits' errors relative to itself, so is every product with a gradient; a root's share of an entry
    # is below w (|x| + 2 |t|) / sqrt(wide) for its own terms and, through the weights of the attention, that times sqrt(dim) T more.
    live = int((dst >= 0).sum())
    share = 1.5 * (X + 2 * T) * wide ** -0.5
    for name, g, r, mass in (("table", grads[0], want[0], share * (1 + dim ** 0.5 * T * T)), ("bias", grads[1], want[1], 1.5),
                             ("age", grads[2], want[2], share * wide ** 0.5 * T)):
        assert float(r.abs().max()) > 1e-3 or (name == "age" and window == 1), name          # (the weight of a single slot is 1 whatever its age)
        assert float((g.double() - r).abs().max()) <= 4 * logit * live * mass, name
    with torch.no_grad():
        assert torch.equal(m.loss(nodes, times, dst) == 0, dst < 0)
    assert m.status() == 0


@pytest.mark.parametrize("dtype,bits", [(F32, 32), (F32, 8), (BF16, 32), (BF16, 8)])
def test_steps_repeat_and_are_those_of_the_parts(workload, dtype, bits):
    """Two models from one seed take the same steps, bit for bit; each is AdamW on the losses' gradients; the 16-bit table is the weights rounded."""
    from paper_2608_16305_b200 import destinations as D
    make = lambda: D.DestinationModel(workload, dtype=dtype, bits=bits, lr=1e-2, weight_decay=0.01, seed=5)
    a, b = make(), make()
    for i in range(4):
        la = a.step(i)
        loss = b.loss(*b.targets(i))
        grads = torch.autograd.grad(loss.sum(), b.leaves)
        b.optimizer.step(list(grads), grad_scale=1.0 / loss.numel())
        assert torch.equal(la, loss.detach())
    for x, y in zip((a.weights, *a.leaves), (b.weights, *b.leaves)):
        assert torch.equal(x, y)
    assert torch.equal(a.table.detach(), a.weights.detach().to(dtype)) and int(a.optimizer.steps[0]) == 4
    assert bool((a.weights.detach() != make().weights.detach()).any()) and a.status() == 0


@pytest.mark.parametrize("dtype,bits", [(F32, 32), (BF16, 8)])
def test_a_captured_step_is_the_eager_one(workload, dtype, bits):
    from paper_2608_16305_b200 import destinations as D
    make = lambda: D.DestinationModel(workload, dtype=dtype, bits=bits, lr=1e-2, seed=7)
    eager, mine = make(), make()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        mine.step(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        loss = mine.step(0)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for _ in range(4):
        want = eager.step(0)
    assert torch.equal(loss, want)
    for x, y in zip((mine.weights, *mine.leaves), (eager.weights, *eager.leaves)):
        assert torch.equal(x, y)


def test_auxiliary_events_take_no_part(stream):
    from paper_2608_16305_b200 import destinations as D
    from paper_2608_16305_b200.trainer import DeviceWorkload
    w = DeviceWorkload(wl.make_stream(wl.scaled(stream.cfg, replay_frac=0.5)), embed_aux=True)
    m = D.DestinationModel(w, seed=1)
    b = next(i for i in range(2, 20) if bool((w.loss_mask(i) == 0).any()) and bool((w.loss_mask(i) != 0).any()))
    mask = w.loss_mask(b) != 0
    src, t, dst = m.targets(b)
    assert torch.equal(dst >= 0, mask)
    loss = m.step(b)
    assert bool((loss[~mask] == 0).all()) and bool((loss[mask] > 0).all()) and bool(torch.isfinite(loss).all())


def test_no_targets(workload):
    from paper_2608_16305_b200 import destinations as D
    m = D.DestinationModel(workload, seed=1)
    none = lambda dt: torch.empty(0, dtype=dt, device="cuda")
    loss = m.loss(none(torch.int32), none(torch.float64), none(torch.int32))
    grads = torch.autograd.grad(loss.sum(), m.leaves, allow_unused=True)
    assert loss.shape == (0,) and bool((grads[0] == 0).all()) and bool((grads[1] == 0).all())
    with torch.no_grad():
        assert m.loss(none(torch.int32), none(torch.float64), none(torch.int32)).shape == (0,)


def test_the_first_call_of_a_thread(workload):
    """A thread that has made no call to the device before (autograd's, say) comes to the library first."""
    import threading
    from paper_2608_16305_b200 import binding as B
    n, rows, dim = 40, 90, 64
    for dtype in (F32, BF16):
        g = torch.Generator(device="cuda").manual_seed(9)
        q, t = (torch.randn((k, dim), generator=g, device="cuda").to(dtype) for k in (n, rows))
        y = torch.arange(n, dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        kept, d = torch.empty(B.destination_loss_kept(n, dim), device="cuda"), torch.ones(n, device="cuda")
        scratch = lambda: torch.empty(B.destination_loss_scratch(n, rows, dim, dtype), dtype=torch.uint8, device="cuda")
        B.destination_loss(q, t, y, torch.empty(n, device="cuda"), scratch(), status, kept=kept)
        here, there, a, b = torch.empty_like(t), torch.zeros_like(t), scratch(), scratch()
        B.destination_loss_backward(q, t, y, kept, d, None, here, a, status)
        torch.cuda.synchronize()
        caught = []

        def work():
            try:
                B.destination_loss_backward(q, t, y, kept, d, None, there, b, status)
            except Exception as e:
                caught.append(e)
        thread = threading.Thread(target=work)
        thread.start()
        thread.join()
        torch.cuda.synchronize()
        assert not caught and torch.equal(here, there), caught
