"""Decay rates that the AdamW step refuses, before anything is launched."""
import pytest

from paper_2608_16305_b200 import binding as B
from tests.test_table_refusals import PTR, _call, _tensor


@pytest.mark.parametrize("b1,b2", [(1 - 1e-9, 0.999), (0.9, 1 - 2.0 ** -25), (1.0, 0.9), (0.9, 2.0), (-1e-30, 0.9)])
def test_rates_that_are_1_in_fp32(b1, b2):
    from paper_2608_16305_b200 import build
    build.build_library()
    rc, msg = _call(B.load_library().tgnn_adamw_step, (B.TgnnAdamwTensor * 1)(_tensor()), 1, 32, PTR, 1e-3, b1, b2, 1e-8, 1.0, 0)
    assert rc == B.TGNN_EINVAL and "beta" in msg
