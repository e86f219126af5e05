"""pb_last_error(NULL): what it returns on the thread that failed and on others (CPU: refused calls only)."""
import threading

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2003_11666_b200 import build
    build.build()
    import paper_2003_11666_b200 as p
    return p.load_library()


def _in_thread(f):
    out = []
    t = threading.Thread(target=lambda: out.append(f()))
    t.start()
    t.join()
    return out[0]


def _create_fails(lib):
    import ctypes as C
    assert lib.pb_mlp_run_static((C.c_int32 * 1)(8), 1, 0.1, 0.9, 3, None, None, None, None, 2, None, None) != 0
    return lib.pb_last_error(None)


def _token_call_fails(lib):
    assert lib.pb_embed_forward(None, 9, 1, 1, 1, None, 4, 1, 1.0, None, 1, None, None) == -1
    return lib.pb_last_error(None)


def test_a_failed_engine_call_can_be_read_from_another_thread(lib):
    # a worker creates, the thread that waits for it reports
    def wait_and_report():                                         # a thread that has no failure of its own
        text = _in_thread(lambda: _create_fails(lib))
        return text, lib.pb_last_error(None)
    text, reported = _in_thread(wait_and_report)
    assert b"pb_mlp_run_static" in text and reported == text
    assert _in_thread(lambda: lib.pb_last_error(None)) == text


def test_a_failed_token_call_is_read_on_its_own_thread(lib):
    assert b"pb_mlp_run_static" in _create_fails(lib)
    assert b"pb_embed_forward" in _in_thread(lambda: _token_call_fails(lib))
    assert b"pb_mlp_run_static" in lib.pb_last_error(None)         # this thread's view has not changed
    assert b"pb_embed_forward" in _token_call_fails(lib)
    _in_thread(lambda: _create_fails(lib))
    assert b"pb_embed_forward" in lib.pb_last_error(None)          # nor by another thread's failure
    assert b"pb_mlp_run_static" in _create_fails(lib)              # the latest of this thread
