"""How much memory the attention's backward asks for (no GPU needed): two floats a row and query head,
and sums of dk and dv that do not grow with the heads' number."""

import pytest

from paper_2609_36246_gb300 import binding as B
from paper_2609_36246_gb300 import build


@pytest.fixture(scope="module")
def size():
    build.build()
    return lambda T, Hq, Hk, D: B.lib().olive_workspace_size(16, T, D, Hk, Hq, 0, 0)


def test_sums_are_bounded(size):
    most = 0
    for T in (1, 128, 129, 511, 512, 513, 1000, 2048, 4999, 16384, 19456, 19457, 100_000, 2**20):
        for Hk in (1, 2, 3, 8, 152, 4096):
            for per in (1, 2, 3, 5, 7, 13, 16, 64, 127, 509, 1024, 4093, 4096):
                if Hk * per > 4096:
                    continue
                for D in (8, 64, 128):
                    total, stats = size(T, Hk * per, Hk, D), 8 * T * Hk * per
                    assert total >= stats and total % 256 == 0
                    most = max(most, total - stats)
    assert 50e6 < most <= 100e6 + 512


def test_parts_where_they_are_worth_a_launch(size):
    for T, Hq, Hk, D, parts in ((100, 8, 1, 64, 1), (512, 8, 1, 64, 8), (5003, 15, 3, 96, 5), (16384, 64, 1, 128, 5),
                                (4096, 32, 4, 128, 4), (19456, 64, 1, 128, 4), (19457, 64, 1, 128, 1), (4096, 9, 1, 64, 9)):
        sums = 8 * parts * T * Hk * D if parts > 1 else 0
        assert 0 <= size(T, Hq, Hk, D) - 8 * T * Hq - sums < 512, (T, Hq, Hk)
