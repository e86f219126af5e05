"""Scratch that is laid out for some rows serves every smaller number of them: a program sizes it once, and its last batch is shorter."""
import pytest

from tests.test_token_refusals import lib  # noqa: F401


def _counts(most):
    """Row counts up to `most`: all small ones, and neighbours of powers of two and of tiles."""
    some = set(range(0, 140)) | {most}
    k = 128
    while k <= most:
        some |= {k - 1, k, k + 1, k + k // 2, 3 * k // 2 + 1}
        k *= 2
    some |= set(range(256, 5000, 256)) | set(range(257, 5000, 256))
    return sorted(n for n in some if 0 <= n <= most)


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("vocab,dim", [(1000, 512), (32000, 1024), (131072, 256), (131072, 128), (50021, 1001), (300, 40), (131072, 4096), (2500, 2048), (1, 1)])
def test_head_sizes_grow_with_the_rows(lib, vocab, dim, dtype, backward):         # noqa: F811
    for aligned in (0, 1):
        sizes = [lib.pb_head_scratch_bytes(dtype, n, vocab, dim, aligned, backward) for n in _counts(20000)]
        assert all(0 < a <= b for a, b in zip(sizes, sizes[1:]))
    # rows that do not start on 16 bytes need no less: of a single row the stride does not count
    for n in _counts(20000):
        assert lib.pb_head_scratch_bytes(dtype, n, vocab, dim, 0, backward) >= lib.pb_head_scratch_bytes(dtype, n, vocab, dim, 1, backward)
