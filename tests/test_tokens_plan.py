"""The splits of linear_lora and moe_layer (csrc/tokens_plan.h, host C++ over sizes
and compute units), compiled here with g++ and checked without a GPU."""
import shutil

import pytest

from qmlp_testutil import host_library

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")

SRC = """
#include "tokens_plan.h"
extern "C" int few_tiles(int n, int cus) { return qmlp::lora_few_tiles(n, cus); }
extern "C" int shares(int M, int n, int k, int cus) { return qmlp::lora_shares(M, n, k, cus); }
extern "C" int large(int M, int n, int cus) { return qmlp::lora_large_tiles(M, n, cus); }
extern "C" int two(int inst, int E, int f, int bits, int cus) { return qmlp::moe_two_tiles(inst, E, f, bits, cus); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return host_library(SRC, tmp_path_factory.mktemp("plan"))


@pytest.mark.parametrize("cus", [32, 64, 128, 256])
def test_shares_fill_the_chip_and_no_more(plan, cus):
    for M in (1, 17, 64, 65, 128, 129, 300, 512, 513, 4096):
        for n in (1, 130, 2560, 6144, 28672):
            for k in (64, 448, 512, 1024, 4096, 17408):
                s, tiles = plan.shares(M, n, k, cus), (M + 127) // 128 * ((n + 127) // 128)
                assert s == 1 or (M <= 512 and s * tiles <= cus and k // 64 // s >= 8)
                assert s > 1 or M > 512 or 2 * tiles > cus or k // 64 < 16


def test_rules_count_the_compute_units_of_the_device(plan):
    """A partition of the chip has fewer places: fewer shares, two tiles a workgroup and large tiles earlier."""
    assert [plan.shares(67, 6144, 4096, c) for c in (32, 64, 128, 256)] == [1, 1, 2, 5]
    assert [plan.few_tiles(2560, c) for c in (128, 256)] == [2, 1]
    assert [plan.large(1024, 6144, c) for c in (64, 256)] == [1, 0]
    assert [plan.two(4, 2, 1536, 4, c) for c in (128, 256)] == [1, 0]
    assert not plan.two(4, 32, 2880, 2, 128) and plan.two(256, 32, 2880, 2, 128)   # 2 bits: from two instances an expert
