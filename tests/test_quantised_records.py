"""Records of the boundary refresh in few bits are smaller than fp32 rows, or the refresh in few bits is refused."""
import numpy as np
import pytest
import torch

from paper_2608_16305_b200 import binding as B
from paper_2608_16305_b200 import distributed as D


class _Cache:
    def __init__(self, rows, heads, dim, bits, device, record):
        self.rows, self.heads, self.dim, self.bits = rows, heads, dim, bits
        # what a record holds: codes padded to 32, 64 or 128 a group, a time, a scale of 2 bytes a group, in steps of 16 bytes
        pad = 32 if dim <= 32 else 64 if dim <= 64 else 128
        self.record_bytes = -(-(heads * pad * bits // 8 + 8 + 2 * heads) // 16) * 16
        self.data = torch.zeros((rows, self.record_bytes), dtype=torch.uint8)


def _plan():
    nodes = torch.zeros((1, 4), dtype=torch.int32)
    return D.RefreshPlan.from_lists(nodes, np.array([[0, 0]]), nodes, np.array([[0, 0]]), 1, 0)


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2608_16305_b200 import build
    build.build_library()


@pytest.mark.parametrize("bits", [8, 4])
def test_records_are_smaller_than_rows_or_refused(bits):
    taken = []
    for d in range(1, 1100):
        groups = [h for h in range(1, d + 1) if d % h == 0 and d // h <= 128]
        worth = min(_Cache(1, h, d // h, bits, None, True).record_bytes for h in groups) < 4 * d + 8
        if not worth:
            with pytest.raises(ValueError, match="record"):
                D.QuantisedRefresh(_plan(), d, bits, cache=_Cache)
            continue
        ref = D.QuantisedRefresh(_plan(), d, bits, cache=_Cache)
        assert ref.send.heads * ref.send.dim == d and ref.send.record_bytes < 4 * d + 8, d
        taken.append(d)
    # widths with a divisor from 16 to 128, among them those of this package, are taken; primes above 128 have groups of one value only
    assert {16, 100, 172, 256, 300, 344} <= set(taken)
    assert not {1, 131, 262, 1031} & set(taken)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("heads,dim", [(1, 100), (3, 100), (4, 32), (2, 33), (5, 128), (131, 1)])
def test_record_bytes(bits, heads, dim):
    assert B.record_bytes(heads, dim, bits, times=True) == _Cache(1, heads, dim, bits, None, True).record_bytes
    code = B.load_library().tgnn_cache_code_bytes(dim, bits)
    assert 0 <= B.record_bytes(heads, dim, bits, times=True) - (heads * code + 8 + 2 * heads) < 16
    assert B.record_bytes(heads, dim, bits, times=False) in (B.record_bytes(heads, dim, bits), B.record_bytes(heads, dim, bits) - 16)


def test_record_bytes_refuses():
    for args in ((0, 10, 4), (1, 129, 4), (1, 10, 5)):
        with pytest.raises(B.TgnnError):
            B.record_bytes(*args)
