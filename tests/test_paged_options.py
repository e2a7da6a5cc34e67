"""Options of the paged attention calls as the binding passes them on."""
import sys

import pytest

from paper_2506_07533_b200 import binding as mq


@pytest.mark.parametrize("window, passed", [(0, 0), (1, 1), (1 << 30, 1 << 30), ((1 << 31) - 1, 1 << 30), (1 << 31, 1 << 30), ((1 << 32) + 5, 1 << 30),
                                            (sys.maxsize, 1 << 30), (-1, -1), (5 - (1 << 32), -1)])
def test_windows_past_32_bits_hide_nothing(window, passed):
    """They lost their upper bits: 2^32 + 5 became a window of 5, the largest integer was refused."""
    assert mq.make_attn_options(window=window).view.window == passed
