"""Rows looked up by id and the table's gradient, against sums in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def half_step(dt):
    return torch.finfo(dt).eps / 2


def tiny(dt):
    """Half the spacing of the type's smallest numbers."""
    return torch.finfo(dt).smallest_normal * torch.finfo(dt).eps / 2


def make(rows, dim, ids, dtype, out_dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    table = torch.randn(rows, dim, generator=g, device="cuda").to(dtype)
    dout = torch.randn(ids.numel(), dim, generator=g, device="cuda").to(out_dtype)
    return table, dout


def both(table, ids, dout, scale, status=None):
    from paper_2608_16305_b200 import binding as B
    rows, dim = table.shape
    status = torch.zeros(1, dtype=torch.int32, device="cuda") if status is None else status
    out = torch.full_like(dout, float("nan"))
    B.lookup(table, ids, out, status, scale=scale)
    dtable = torch.full_like(table, float("nan"))
    scratch = torch.full((B.lookup_scratch(ids.numel(), rows, dim),), 0xFF, dtype=torch.uint8, device="cuda")
    B.lookup_backward(ids, dout, dtable, scratch, status, scale=scale)
    return out, dtable, status


def check(table, ids, dout, scale, out, dtable):
    rows, dim = table.shape
    flat = ids.reshape(-1).long()
    ok = (flat >= 0) & (flat < rows)
    used = flat[ok]
    ref = torch.zeros(flat.numel(), dim, dtype=torch.float64, device="cuda")
    ref[ok] = table.double()[used] * float(np.float32(scale))
    # one product in fp32 and one rounding to the output's type
    e = (out.reshape(-1, dim).double() - ref).abs()
    lim = ref.abs() * (2.0 ** -24 + half_step(out.dtype) * (1 + 2.0 ** -23)) + tiny(out.dtype)
    assert bool((e <= lim).all()), float((e - lim).max())
    x = dout.double()[ok]
    s = torch.zeros(rows, dim, dtype=torch.float64, device="cuda").index_add_(0, used, x)
    a = torch.zeros(rows, dim, dtype=torch.float64, device="cuda").index_add_(0, used, x.abs())
    k = torch.bincount(used, minlength=rows)[:, None].double()
    f = float(np.float32(scale))
    # k terms added in fp32 in any order: k - 1 roundings of at most half a step of a partial sum, and that of the product
    lim = k * 2.0 ** -24 * 1.001 * a * abs(f) + s.abs() * abs(f) * half_step(dtable.dtype) * 1.001 + tiny(dtable.dtype)
    e = (dtable.double() - s * f).abs()
    assert bool((e <= lim).all()), float((e - lim).max())
    assert bool((dtable[k[:, 0] == 0] == 0).all())


@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in (F32, BF16, F16) for b in (F32, BF16, F16)])
@pytest.mark.parametrize("rows,dim,n", [(1, 1, 1), (7, 25, 300), (1000, 32, 6000), (300, 101, 20_000), (70_000, 50, 33_000)])
def test_against_64_bits(dtype, out_dtype, rows, dim, n):
    g = torch.Generator(device="cuda").manual_seed(rows + n)
    ids = (torch.rand(n, generator=g, device="cuda") ** 3 * rows).long().clamp(max=rows - 1)      # the first rows are hubs
    ids = torch.where(torch.rand(n, generator=g, device="cuda") < 0.1, torch.full_like(ids, -1), ids).to(torch.int32)
    table, dout = make(rows, dim, ids, dtype, out_dtype)
    out, dtable, status = both(table, ids, dout, 1.7)
    check(table, ids, dout, 1.7, out, dtable)
    assert int(status.item()) == 0


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 1023, 1024, 1025, 8191, 8192, 8193, 65_537, 300_001, 1_200_000])
@pytest.mark.parametrize("kind", ["one", "ascending", "random", "unused"])
def test_lengths_and_orders(n, kind):
    rows, dim = 513, 8
    at = torch.arange(n, device="cuda")
    ids = {"one": torch.full_like(at, 5), "ascending": at * rows // n, "random": (at * 7919) % rows, "unused": torch.full_like(at, -1)}[kind]
    table, dout = make(rows, dim, ids, F32, F32, seed=n)
    out, dtable, _ = both(table, ids, dout, 0.5)
    check(table, ids, dout, 0.5, out, dtable)


@pytest.mark.parametrize("rows", [1, 2, 127, 128, 255, 256, 257, 65_535, 65_536, 65_537, 1 << 24])
@pytest.mark.parametrize("n", [900, 20_000])
def test_tables_at_the_digits_borders(rows, n):
    g = torch.Generator(device="cuda").manual_seed(rows)
    ids = torch.randint(0, rows, (n,), generator=g, device="cuda")
    ids[0], ids[-1], ids[n // 2] = rows - 1, 0, -7
    table, dout = make(rows, 4, ids, BF16, F32)
    out, dtable, _ = both(table, ids, dout, 1.0)
    check(table, ids, dout, 1.0, out, dtable)


@pytest.mark.parametrize("dim", [1, 2, 3, 8, 33, 64, 127, 128, 172, 256, 511, 1000, 8192])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_widths(dim, dtype):
    g = torch.Generator(device="cuda").manual_seed(dim)
    ids = torch.randint(-1, 40, (5, 130), generator=g, device="cuda", dtype=torch.int32)
    table, dout = make(40, dim, ids, dtype, dtype)
    out, dtable, _ = both(table, ids, dout, -2.0)
    check(table, ids, dout, -2.0, out, dtable)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("offset", [1, 2, 3])
def test_addresses_between_words(dtype, offset):
    """Tables, rows and gradients that begin inside a 16-byte word."""
    from paper_2608_16305_b200 import binding as B
    rows, dim, n = 50, 64, 20_000
    cut = lambda r: torch.full((r * dim + 8,), 9.0, dtype=dtype, device="cuda")
    bufs = [cut(rows), cut(n), cut(n), cut(rows)]
    table, dout, out, dtable = (b[offset:offset + (b.numel() - 8)].view(-1, dim) for b in bufs)
    g = torch.Generator(device="cuda").manual_seed(1)
    table.copy_(torch.randn(rows, dim, generator=g, device="cuda"))
    dout.copy_(torch.randn(n, dim, generator=g, device="cuda"))
    ids = torch.randint(-2, rows - 5, (n,), generator=g, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.lookup(table, ids, out, status, scale=3.0)
    scratch = torch.empty(B.lookup_scratch(n, rows, dim), dtype=torch.uint8, device="cuda")
    B.lookup_backward(ids, dout, dtable, scratch, status, scale=3.0)
    check(table, ids, dout, 3.0, out, dtable)
    for b, x in zip(bufs, (table, dout, out, dtable)):           # what lies around is left as it was
        assert bool((b[:offset] == 9).all()) and bool((b[offset + x.numel():] == 9).all())


def test_ids_beyond_the_table_are_zeros_and_reported():
    ids = torch.tensor([0, 3, 4, -1, 2**31 - 1, 2], dtype=torch.int32, device="cuda")
    table, dout = make(4, 16, ids, F32, F32)
    out, dtable, status = both(table, ids, dout, 1.0)
    check(table, ids, dout, 1.0, out, dtable)
    assert int(status.item()) == 4
    big = torch.tensor([2**40, 1, -(2**50)], device="cuda")
    table, dout = make(4, 16, big, F32, F32)
    out, dtable, status = both(table, big, dout, 1.0)
    check(table, big, dout, 1.0, out, dtable)
    assert int(status.item()) == 4


def test_unused_slots_take_nothing_from_their_rows():
    """A gradient of an unused slot may be anything; a row that no id names may be too."""
    ids = torch.tensor([1, -1, 0, -1], dtype=torch.int32, device="cuda")
    table, dout = make(3, 20, ids, F32, F32)
    table[2] = float("nan")
    dout[1], dout[3] = float("nan"), float("inf")
    out, dtable, _ = both(table, ids, dout, 1.0)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(dtable).all())
    assert bool((dtable[2] == 0).all()) and torch.equal(dtable[0], dout[2]) and torch.equal(dtable[1], dout[0])


def test_no_ids_and_no_rows():
    from paper_2608_16305_b200 import binding as B
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    table = torch.randn(5, 6, device="cuda")
    B.lookup(table, none, torch.empty(0, 6, device="cuda"), status)
    d = torch.ones(5, 6, device="cuda")
    B.lookup_backward(none, torch.empty(0, 6, device="cuda"), d, torch.empty(B.lookup_scratch(0, 5, 6), dtype=torch.uint8, device="cuda"), status)
    assert bool((d == 0).all())
    ids = torch.tensor([-1, -1], device="cuda")
    out = torch.ones(2, 6, device="cuda")
    B.lookup(torch.empty(0, 6, device="cuda"), ids, out, status)
    assert bool((out == 0).all()) and int(status.item()) == 0
    B.lookup_backward(ids, out, torch.empty(0, 6, device="cuda"), torch.empty(B.lookup_scratch(2, 0, 6), dtype=torch.uint8, device="cuda"), status)


def test_the_same_bits_every_time_and_from_a_graph_on_another_stream():
    from paper_2608_16305_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(3)
    for n in (9000, 100_000):
        ids = (torch.rand(n, generator=g, device="cuda") ** 4 * 3000).int()
        table, dout = make(3000, 100, ids, F32, F32)
        out, first, status = both(table, ids, dout, 1.0)
        scratch = torch.empty(B.lookup_scratch(n, 3000, 100), dtype=torch.uint8, device="cuda")
        again = torch.empty_like(first)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            B.lookup(table, ids, out, status)
            B.lookup_backward(ids, dout, again, scratch, status)
        for _ in range(3):
            again.fill_(7)
            out.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(first, again)
        check(table, ids, dout, 1.0, out, again)


def test_gradients_under_autograd():
    from paper_2608_16305_b200 import destinations as D
    g = torch.Generator(device="cuda").manual_seed(4)
    table = torch.randn(30, 12, generator=g, device="cuda").requires_grad_()
    ids = torch.randint(-1, 30, (17, 5), generator=g, device="cuda", dtype=torch.int32)
    w = torch.randn(17, 5, 12, generator=g, device="cuda")
    out = D.lookup(table, ids, scale=2.0, dtype=torch.bfloat16)
    assert out.shape == (17, 5, 12) and out.dtype == torch.bfloat16
    (out.float() * w).sum().backward()
    check(table.detach(), ids, w.bfloat16().view(-1, 12), 2.0, out.detach(), table.grad)
    # a column taken of a wider gradient, and a table that is a view
    wide = torch.randn(12, 30, generator=g, device="cuda").requires_grad_()
    out = D.lookup(wide.t(), ids)
    out[:, :, ::2].sum().backward()
    assert wide.grad.shape == (12, 30) and bool((wide.grad[1::2] == 0).all())
    counts = torch.bincount(ids[ids >= 0].long(), minlength=30).float()
    assert torch.equal(wide.grad[0], counts)


@pytest.mark.parametrize("n,rows", [(50, 1), (50, 3), (50, 4), (50, 9), (1000, 33), (8192, 8191), (8192, 8192), (8192, 8193), (8193, 8191), (4096, 16_384), (4096, 16_383),
                                    (4097, 16_384), (64, 16_384), (64, 16_385)])
@pytest.mark.parametrize("dim,dtype", [(36, F32), (34, F32), (33, BF16), (72, BF16)])
def test_few_ids_over_few_rows(n, rows, dim, dtype):
    g = torch.Generator(device="cuda").manual_seed(n + rows)
    ids = torch.randint(-1, rows, (n,), generator=g, device="cuda")
    ids[::5] = rows - 1
    ids[n // 2], ids[0] = (1 << 33) + 1, -(1 << 33)
    table, dout = make(rows, dim, ids, dtype, dtype)
    out, dtable, status = both(table, ids, dout, 1.0)
    check(table, ids, dout, 1.0, out, dtable)
    assert int(status.item()) == 4
    assert torch.equal(both(table, ids, dout, 1.0)[1], dtable)


@pytest.mark.parametrize("n,dim", [(70_001, 100), (140_001, 100), (530_001, 100), (530_001, 128), (530_001, 33)])
@pytest.mark.parametrize("kind", ["hubs", "even"])
def test_chunks_of_every_size(n, dim, kind):
    g = torch.Generator(device="cuda").manual_seed(n + dim)
    at = torch.rand(n, generator=g, device="cuda")
    ids = ((at ** 6 if kind == "hubs" else at) * 700).long().clamp(max=699)
    table, dout = make(700, dim, ids, F32, F32)
    out, dtable, _ = both(table, ids, dout, 1.0)
    check(table, ids, dout, 1.0, out, dtable)
