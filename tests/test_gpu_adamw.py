"""The AdamW step over many tensors: parameters against 64 bits, 8-bit states against their definition bit by bit."""
import math

import numpy as np
import pytest
import torch

from oracle import adamw as oa

pytestmark = pytest.mark.gpu
LR, B1, B2, EPS = 3e-3, 0.9, 0.999, 1e-8


def make(sizes, bits, dtype=torch.float32, seed=0, **kw):
    from paper_2608_16305_b200 import destinations as D
    g = torch.Generator(device="cuda").manual_seed(seed)
    params = [torch.randn(s, generator=g, device="cuda") for s in sizes]
    opt = D.AdamW(params, lr=LR, betas=(B1, B2), eps=EPS, bits=bits, seed=77, **kw)
    grads = lambda: [(torch.randn(s, generator=g, device="cuda") * torch.exp(3 * torch.randn(s, generator=g, device="cuda")) * 1e-2).to(dtype)
                     for s in sizes]
    return params, opt, grads


def host(x):
    return x.detach().float().cpu().numpy()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sizes", [[1], [255], [256], [257], [2048, 3, 0, 2049, 70_001], [5] * 41, list(range(1, 401))])
def test_steps_against_the_definition(sizes, dtype, bits):
    decay = [0.1 * (i % 3) for i in range(len(sizes))]
    params, opt, grads = make(sizes, bits, dtype, weight_decay=decay)
    state = [oa.State(s, bits) for s in sizes]
    for t in range(1, 4):
        g = grads()
        before = [host(p).astype(np.float64) for p in params]
        opt.step(g, grad_scale=0.25)
        for i, s in enumerate(sizes):
            new, most = oa.step(state[i], before[i], host(g[i]), t, i, LR, B1, B2, EPS, decay[i], 0.25, 77)
            # The two parts of m are rounded before they are added, so their error is a part of |b1 m| + |(1 - b1) g|, which m falls below by any factor
            # where they cancel.  Half steps of 2^-24 on the way: g 1, parts and sum of m 2, v (3 half steps) and its root 2.5, the corrections 2, product
            # and sum below 2, the quotient 4 (2^-22), decay, sum and lr 3: below 17; then the parameter's own rounding
            lim = most * 17 * 2.0 ** -24 + np.abs(new) * 2.0 ** -24 * 1.001
            assert (np.abs(host(params[i]) - new) <= lim + 1e-12).all(), (t, i)
        got = opt.moments()
        for i in range(len(sizes)):
            assert np.array_equal(host(got[0][i]), state[i].m) and np.array_equal(host(got[1][i]), state[i].v), (t, i)
        if bits == 8:
            for i in range(len(sizes)):
                assert np.array_equal(opt.m[i].cpu().numpy(), state[i].cm) and np.array_equal(opt.v[i].cpu().numpy(), state[i].cu)
        assert opt.steps.tolist() == [t, 0]


def test_many_tensors_take_several_launches():
    sizes = [1 + i % 5 for i in range(1000)]
    params, opt, grads = make(sizes, 32)
    g = grads()
    before = [p.clone() for p in params]
    opt.step(g)
    assert opt.steps.tolist() == [1, 0]
    for i in (0, 359, 360, 719, 720, 999):
        # at the first step the moments' corrections cancel: the step is lr * g / (|g| + eps)
        want = before[i].double() - LR * g[i].double() / (g[i].double().abs() + EPS)
        assert float((params[i].double() - want).abs().max()) <= 4 * LR * 2.0 ** -22 + float(before[i].abs().max()) * 2.0 ** -23


@pytest.mark.parametrize("bits", [8, 32])
def test_copies_and_missing_gradients(bits):
    sizes = [300, 4097, 17]
    copies = [torch.empty(300, dtype=torch.bfloat16, device="cuda"), None, torch.empty(17, dtype=torch.float16, device="cuda")]
    params, opt, grads = make(sizes, bits, copies=copies)
    g = grads()
    g[1] = None
    before = params[1].clone()
    opt.step(g)
    assert torch.equal(params[1], before) and int(opt.v[1].sum()) == 0
    assert torch.equal(copies[0], params[0].bfloat16()) and torch.equal(copies[2], params[2].half())
    for p, x in zip(params, grads()):
        p.requires_grad_()
        p.grad = x
    opt.step()
    assert opt.steps.tolist() == [2, 0] and not torch.equal(params[1].detach(), before)


@pytest.mark.parametrize("offset", [1, 2, 3])
@pytest.mark.parametrize("bits", [8, 32])
def test_addresses_between_words(offset, bits):
    from paper_2608_16305_b200 import destinations as D
    n = 1111
    g = torch.Generator(device="cuda").manual_seed(8)
    pb, gb = torch.randn(n + 8, generator=g, device="cuda"), torch.randn(n + 8, generator=g, device="cuda")
    whole = pb.clone()
    p, x = pb[offset:offset + n], gb[offset:offset + n]
    other = p.clone()
    a, b = D.AdamW([p], bits=bits, seed=5), D.AdamW([other], bits=bits, seed=5)
    for _ in range(2):
        a.step([x])
        b.step([x.clone()])
    assert torch.equal(p, other) and torch.equal(a.moments()[1][0], b.moments()[1][0])
    assert torch.equal(pb[:offset], whole[:offset]) and torch.equal(pb[offset + n:], whole[offset + n:])


def test_zero_and_extreme_gradients_in_8_bits():
    n = 1024
    params, opt, _ = make([n], 8)
    state = oa.State(n, 8)
    x = np.zeros(n, np.float32)
    x[256:512] = 1e-30                                   # a block below 2^-60 is held as zeros
    x[512:768] = np.float32(1e4) ** np.linspace(-4, 4, 256, dtype=np.float32)
    x[768] = 3.0                                         # one value among zeros
    for t in (1, 2):
        before = host(params[0]).astype(np.float64)
        opt.step([torch.from_numpy(x).cuda()])
        new, most = oa.step(state, before, x, t, 0, LR, B1, B2, EPS, 0.0, 1.0, 77)
        assert np.isfinite(host(params[0])).all()
        assert np.array_equal(opt.m[0].cpu().numpy(), state.cm) and np.array_equal(opt.v[0].cpu().numpy(), state.cu)
    assert (state.cu[:512] == 0).all() and (state.cu[512:768] >= 1).all()


def test_a_block_with_an_infinity_reads_back_as_nan_and_no_other():
    params, opt, _ = make([600], 8)
    x = torch.ones(600, device="cuda")
    x[300] = float("inf")
    opt.step([x])
    m, v = opt.moments()
    for y in (m[0], v[0]):
        assert bool(torch.isnan(y[256:512]).all()) and bool(torch.isfinite(y[:256]).all()) and bool(torch.isfinite(y[512:]).all())


def test_a_decaying_second_moment_follows_its_mean():
    """Rounded by chance, u = sqrt(v) without gradients falls as it would in 32 bits; to the nearest it would never move."""
    n = 1 << 16
    params, opt, _ = make([n], 8)
    opt.step([torch.full((n,), 1.0, device="cuda")])
    top = torch.zeros(n, device="cuda")
    top[::256] = 1.0                                     # keeps every block's scale
    before = opt.moments()[1][0].clone()
    steps = 60
    for _ in range(steps):
        opt.step([top])
    u = opt.moments()[1][0].view(-1, 256)[:, 1:].sqrt().double()
    want = float(before[1].sqrt()) * B2 ** (steps / 2)
    # a step's rounding has a spread of at most one code, 2 / 255 of the top's u; 60 steps of 65 280 values: the mean's is sqrt(60 / 65280) of that, taken five times
    assert abs(float(u.mean()) - want) <= 5 * math.sqrt(steps / u.numel()) * (2 / 255) * float(u.max())


@pytest.mark.parametrize("bits", [8, 32])
def test_captured_and_replayed(bits):
    params, opt, grads = make([3000, 70], bits)
    twin_p, twin, _ = make([3000, 70], bits)
    g = grads()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        opt.step(g)
    for _ in range(4):
        graph.replay()
        twin.step(g)
    torch.cuda.synchronize()
    assert opt.steps.tolist() == twin.steps.tolist() == [4, 0]
    for a, b in zip(params + opt.m + opt.v, twin_p + twin.m + twin.v):
        assert torch.equal(a, b)


def test_many_values_in_8_bits():
    """So many values that a thread block takes more of them."""
    test_steps_against_the_definition([9_800_001, 300, 4097], torch.bfloat16, 8)
