"""Errors of lookups and destination losses that were given no status tensor."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_an_index_beyond_its_table_can_be_read_afterwards():
    from paper_2608_16305_b200 import destinations as D
    D.status(clear=True)
    table = torch.randn(30, 16, device="cuda")
    q = torch.randn(3, 16, device="cuda")
    ok, bad = torch.tensor([0, -1, 29], device="cuda"), torch.tensor([0, 30, 2], device="cuda")
    other = torch.cuda.Stream()
    for call in (lambda i: D.lookup(table, i), lambda i: D.destination_loss(q, table, i)):
        call(ok)
        assert D.status() == 0
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            call(bad)
        torch.cuda.synchronize()
        assert D.status() == D.status(0) == D.status("cuda:0") == 4
        call(ok)
        assert D.status(clear=True) == 4 and D.status() == 0
        with torch.inference_mode():
            call(bad)
        assert D.status(clear=True) == 4
    mine = torch.zeros(1, dtype=torch.int32, device="cuda")
    D.lookup(table, bad, status=mine)
    assert int(mine) == 4 and D.status() == 0


def test_captured_calls_without_a_status():
    from paper_2608_16305_b200 import destinations as D
    table, ids = torch.randn(30, 16, device="cuda"), torch.tensor([5, 1], device="cuda")
    D.status(clear=True)
    held = dict(D._flags)
    for first in (True, False):                          # before any other call of the process, and behind others
        D._flags.clear()
        if not first:
            D.lookup(table, ids)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = D.lookup(table, ids)
        assert len(D._flags) == (0 if first else 1)
        ids[0] = 30
        graph.replay()
        torch.cuda.synchronize()
        assert bool((out[0] == 0).all()) and torch.equal(out[1], table[1])
        assert D.status() == (0 if first else 4)
        ids[0] = 5
    D._flags.clear()
    D._flags.update(held)
