"""Sizes next to 2^31 are refused where blocks of 128 rows or columns would not fit an int; no GPU is needed."""
import ctypes

import pytest

from paper_2311_00368_b200 import build as b2sp_build

OK, INVALID, UNSUPPORTED = 0, 1, 2
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def b():
    b2sp_build.build()
    from paper_2311_00368_b200 import binding
    return binding


@pytest.mark.parametrize("M, K", [(MOST, 8), (MOST - 126, 8), (8, MOST), (8, MOST - 126), (MOST, MOST), (8, 128 * 32768 + 1)])
def test_plans(b, M, K):
    assert b.lib.b2sp_attention_plan_bytes(1, M, K, 4, 1) == 0
    n = ctypes.c_longlong(0)
    assert b.lib.b2sp_attention_count_tiles(1, M, K, 4, 4096, M + 1, 4096, 1 << 20, 256, ctypes.byref(n), None) == UNSUPPORTED
    assert b.lib.b2sp_attention_prepare(1, M, K, 4, 4096, M + 1, 4096, 1, 1 << 20, 1 << 50, None) == UNSUPPORTED


def test_the_largest_plans(b):
    assert b.lib.b2sp_attention_plan_bytes(1, MOST - 127, 8, 4, 1) > 4 * (MOST - 127) // 128
    assert b.lib.b2sp_attention_plan_bytes(1, 8, 128 * 32768, 4, 1) > 4 * 128 * 32768


@pytest.mark.parametrize("M, K", [(MOST, 8), (8, MOST)])
def test_problems(b, M, K):
    make = lambda plan: b._PROBLEM(1, 1, 1, M, K, 1, 1, 1.0, 4096, M + 1, 8192, 8, plan, 1 if plan else 0)  # noqa: E731
    x, y = b._HEADS(1 << 20, 1, 0, 0), b._HEADS(1 << 20, 1, 0, 0)
    for suffix in ("", "_bf16"):
        need = getattr(b.lib, "b2sp_attention_workspace_bytes" + suffix)
        assert 512 <= need(make(0), 0) < 1 << 20 if M == MOST else need(make(0), 0) >= 512     # row kernels: any size
        assert need(make(0), 1) == need(make(1 << 20), 0) == need(make(1 << 20), 1) == 0       # with a plan, which there is none of
        assert getattr(b.lib, "b2sp_attention" + suffix)(make(1 << 20), x, y, y, x, 4096, 1 << 20, 1 << 60, 0, None) == UNSUPPORTED
        assert getattr(b.lib, "b2sp_attention_backward" + suffix)(make(1 << 20), x, y, y, x, 4096, x, x, y, y, 1 << 20, 1 << 60, 0, None) == UNSUPPORTED
