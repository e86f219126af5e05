"""Overlaps of the embedding's buffers that are refused, on any machine (tests/test_token_refusals.py has the others)."""
import pytest

from tests.test_token_refusals import ARG, _embed_backward, _embed_forward, lib  # noqa: F401


@pytest.mark.parametrize("change", [dict(ids=1 << 31), dict(ids=(1 << 31) + 10 * 64 * 2 - 8), dict(ids=(1 << 31) - 72)])
def test_embed_forward_refuses_ids_inside_the_output(lib, change):       # noqa: F811
    assert _embed_forward(lib, **change) == ARG
    assert b"overlaps the ids" in lib.pb_last_error(None)


# ids: 40 bytes; scratch: 1 << 20 bytes at 1 << 32; dtable: 100 rows of 256 bytes at 1 << 31; status: 4 bytes
@pytest.mark.parametrize("change", [dict(ids=1 << 32), dict(ids=(1 << 32) + (1 << 20) - 4), dict(ids=(1 << 32) - 36), dict(ids=1 << 31),
                                    dict(ids=(1 << 31) + 100 * 256 - 4), dict(status=1 << 32), dict(status=(1 << 32) + 4096), dict(status=(1 << 30) + 36)])
def test_embed_backward_refuses_ids_and_status_inside_what_it_writes(lib, change):       # noqa: F811
    assert _embed_backward(lib, **change) == ARG
    assert b"buffers overlap" in lib.pb_last_error(None)
