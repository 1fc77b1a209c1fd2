"""Places of events' entries in a T-CSR: event by event, two each; a T-CSR that does not number its events so is refused, not answered wrongly."""
import numpy as np
import pytest
import torch

from paper_2608_16305_b200 import history as H
from paper_2608_16305_b200 import workload as wl


def _history(eid):
    h = H.EventHistory.__new__(H.EventHistory)                     # what places() needs: no cache, no device
    h.eid, h._places = torch.as_tensor(eid, dtype=torch.int32), None
    return h


def _stream_eids(events, seed=0):
    rng = np.random.default_rng(seed)
    src, dst = rng.integers(0, 20, events), rng.integers(0, 20, events)      # (some events join a node to itself)
    return wl.build_tcsr(src.astype(np.int32), dst.astype(np.int32), np.sort(rng.random(events)), 20)[2]


@pytest.mark.parametrize("base", [0, 1, 5000])
def test_places_of_a_stream_and_of_a_part_of_one(base):
    eid = _stream_eids(150) + base
    h = _history(eid)
    for a, b in ((0, 10), (10, 11), (11, 11), (140, 150), (0, 150)):
        at = h.places(base + a, base + b)
        assert torch.equal(h.eid[at], (base + torch.arange(a, b, dtype=torch.int32)).repeat_interleave(2))
        assert len(set(at.tolist())) == 2 * (b - a)
    # events before the first and behind the last have no entries
    assert h.places(base + 145, base + 400).numel() == 10 and h.places(base + 150, base + 160).numel() == 0
    assert h.places(base - 10, base + 2).numel() == 4 and h.places(base - 10, base - 2).numel() == 0 and h.places(base + 9, base + 3).numel() == 0


@pytest.mark.parametrize("what", ["gap", "one entry", "three entries", "odd"])
def test_other_numberings_are_refused(what):
    eid = _stream_eids(60)
    if what == "gap":
        eid = np.where(eid >= 30, eid + 1, eid)
    elif what == "one entry":
        eid = np.delete(eid, [np.nonzero(eid == 7)[0][0], np.nonzero(eid == 9)[0][0]])
    elif what == "three entries":
        eid = np.concatenate([eid, [7, 9]])
    else:
        eid = np.delete(eid, [5])
    h = _history(eid)
    for _ in range(2):
        with pytest.raises(ValueError):
            h.places(0, 5)


def test_no_events():
    assert _history([]).places(0, 3).numel() == 0
