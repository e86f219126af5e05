"""Joins from two host threads at once, whose rows need rings of different sizes."""
import ctypes as C
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def _state(rows, dim):
    """A gradient's tensors, and the C call of it."""
    from paper_2003_11666_b200.binding import load_library, pb_join_args, pb_join_grads
    import paper_2003_11666_b200 as p
    g = torch.Generator(device="cuda").manual_seed(dim)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    b = lambda: rand(rows, dim).to(torch.bfloat16)                 # noqa: E731
    s = dict(u=b(), y=b(), dy=b(), dh=b(), w=rand(dim), r=rand(rows).abs(), dx=b(), du=b(),
             s=torch.empty(p.join_scratch_bytes(rows, dim), device="cuda", dtype=torch.uint8))
    at = {k: t.data_ptr() for k, t in s.items()}
    a = pb_join_args(rows=rows, dim=dim, dtype=1, stream_dtype=1, weight_dtype=0, residual_scale=1.0, u=at["u"], ld_u=dim, rows_per_gate=1, post_weight=at["w"],
                     pre_weight=at["w"], y=at["y"], ld_y=dim, rstd_post=at["r"], rstd_pre=at["r"])
    d = pb_join_grads(dy=at["dy"], ld_dy=dim, dh=at["dh"], ld_dh=dim, dx=at["dx"], ld_dx=dim, du=at["du"], ld_du=dim)
    lib, n = load_library(), s["s"].numel()
    ra, rd, keep = C.byref(a), C.byref(d), (s, a, d)
    return s, lambda stream: (keep, lib.pb_join_backward(ra, rd, at["s"], n, stream))[1]


def test_two_threads_with_rings_of_their_own():
    rows, turns, failed = 700, 20000, []
    states = [_state(rows, dim) for dim in (6144, 8192)]          # three rows of 61440 bytes in the ring, two of 81920
    want = []
    for s, call in states:
        assert call(torch.cuda.current_stream().cuda_stream) == 0
        want.append((s["dx"].clone(), s["du"].clone()))
    torch.cuda.synchronize()

    def work(call):
        stream = torch.cuda.Stream()
        for k in range(turns):
            if call(stream.cuda_stream) != 0:
                failed.append(k)
            if k % 200 == 199:
                stream.synchronize()
        stream.synchronize()
    threads = [threading.Thread(target=work, args=(call,)) for _, call in states]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, len(failed)
    for (s, _), (dx, du) in zip(states, want):
        assert torch.equal(s["dx"], dx) and torch.equal(s["du"], du)
