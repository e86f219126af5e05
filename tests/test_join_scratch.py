"""Scratch of a join's gradient that is laid out for some rows serves every smaller number of them."""
import itertools

import pytest

from tests.test_head_scratch import _counts
from tests.test_token_refusals import lib  # noqa: F401


@pytest.mark.parametrize("dim", [1, 16, 40, 256, 1000, 1024, 4096, 16384])
@pytest.mark.parametrize("per", [0, 1, 2, 3, 9, 36, 512, 1000, 2048, 1 << 29])
def test_join_sizes_grow_with_the_rows(lib, dim, per):            # noqa: F811
    counts = sorted(set(_counts(70000)) | {k * n + j for n, k, j in itertools.product((444, 888, 1184, 3552, 7104, 14208), (1, 2, 3, 4), (-1, 0, 1))})
    sizes = [lib.pb_join_scratch_bytes(n, dim, per) for n in counts]
    assert all(0 < a <= b for a, b in zip(sizes, sizes[1:]))


def test_a_single_gate_for_all_rows_is_a_gate_of_any_length_that_reaches_them(lib):           # noqa: F811
    for rows in (1, 5, 100, 7105, 20000):
        assert lib.pb_join_scratch_bytes(rows, 64, rows) == lib.pb_join_scratch_bytes(rows, 64, 1 << 30)
