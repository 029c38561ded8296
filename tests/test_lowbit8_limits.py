"""Sizes past what a launch holds are refused as the header says, before anything is launched (no GPU)."""
import pytest

from tests.test_lowbit8_abi import MOST, SHAPE, backward, product


@pytest.mark.parametrize("call,sizes", [
    (backward, dict(rows=3355443, cols=8193, gs=8193)),                 # 5 * 3355443 = 2^24 - 1
    (backward, dict(rows=3355443, cols=10240, gs=10240, gated=1)),
    (backward, dict(rows=2, cols=2 ** 23 + 1, gs=2 ** 24)),
    (backward, dict(rows=4096, cols=2 ** 23, gs=2 ** 23)),
    (product, dict(rows=MOST, out=2 ** 17)),                            # 16384 * 512 tiles
    (product, dict(rows=MOST, cin=131071, out=2 ** 24)),
    (product, dict(rows=2 ** 15, cin=16, out=2 ** 24)),
])
def test_sizes_past_a_launch(call, sizes):
    assert call(**sizes) == SHAPE
