"""The window of kv_attention (csrc/kv_window.h, plain C++), compiled here with g++ and checked without a GPU."""
import shutil

import pytest

from qmlp_testutil import host_library

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")

SRC = """
#include "kv_window.h"
extern "C" int first(int pos, int window) { return qmlp::first_seen(pos, window); }
"""
MOST = 2 ** 31 - 1


def test_every_window_and_position(tmp_path):
    """Positions from a request without cached tokens and with the most new ones to the longest cache; windows to the largest
    int.  What the kernels read lies at or behind the first token seen, in steps of 128 and 32 steps ahead."""
    first = host_library(SRC, tmp_path).first
    places = (0, 1, 2, 15, 16, 127, 128, 129, 4096, 1 << 20, (1 << 20) + 1, (1 << 30) - 1, 1 << 30)
    for pos in [p * s for p in places for s in (1, -1)]:
        for window in sorted({0, 1, 2, MOST, MOST - 1, MOST - 4096, MOST - (1 << 20)} | {p + d for p in places for d in (-1, 0, 1) if p + d > 0}):
            got = first(pos, window)
            assert got == (max(0, pos - window + 1) if window else 0), (pos, window)
            assert 0 <= got <= max(pos, 0) and got // 128 * 128 + 33 * 128 <= MOST
