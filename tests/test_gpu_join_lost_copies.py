"""A row whose copies do not come in time is NaN, and so is what depends on it: no stale numbers leave the joins' kernels.  Nothing faults or
hangs: the waits' limit is a parameter of the kernels, and with a limit of zero they do not wait (the copies land all the same)."""
import ctypes as C
import os
import subprocess

import pytest
import torch

pytestmark = pytest.mark.gpu

WAIT = 200_000_000


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    from paper_2003_11666_b200 import build
    so = str(tmp_path_factory.mktemp("lost") / "lost.so")
    here = os.path.join(os.path.dirname(os.path.abspath(__file__)), "join_lost_copies.cu")
    subprocess.run([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-o", so, here], check=True)
    lib = C.CDLL(so)
    vp = C.c_void_p
    lib.forward.argtypes = [C.c_int, C.c_int] + [vp] * 8 + [C.c_longlong]
    lib.backward.argtypes = [C.c_int, C.c_int] + [vp] * 14 + [C.c_longlong]
    return lib


def _at(t):
    return None if t is None else t.data_ptr()


@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("rows,blocks", [(1, 1), (50, 4), (700, 148)])
def test_forward(kernels, rows, blocks, post, pre):
    import paper_2003_11666_b200 as p
    g = torch.Generator(device="cuda").manual_seed(rows)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    x, u = (rand(rows, 4096).to(torch.bfloat16) for _ in range(2))
    a, b = rand(4096) if post else None, rand(4096) if pre else None
    out = []
    for wait in (WAIT, 0):
        y, h = torch.zeros_like(x), torch.zeros_like(x)
        rp, rr = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
        torch.cuda.synchronize()
        assert kernels.forward(rows, blocks, _at(x), _at(u), _at(a), _at(b), _at(y), _at(h) if pre else None, _at(rp) if post else None, _at(rr) if pre else None, wait) == 0
        out.append((y, h if pre else None, rp if post else None, rr if pre else None))
    ref = [torch.zeros_like(t) if t is not None else None for t in out[0]]
    p.join_forward(x, u, ref[0], h=ref[1], pre_weight=b, post_weight=a, rstd_post=ref[2], rstd_pre=ref[3])
    tol = {torch.bfloat16: 2.0 ** -7, torch.float32: 2.0 ** -18}   # a step of the type: rows of other layouts are summed in another order
    for got, want, lost in zip(out[0], ref, out[1]):
        if got is not None:
            assert bool(((got.double() - want.double()).abs() <= tol[got.dtype] * want.double().abs() + 2.0 ** -18).all())
            assert bool(lost.isnan().all())


@pytest.mark.parametrize("post,dh_,dy_,gate_", [(True, True, True, True), (True, True, False, False), (False, True, True, False), (False, False, True, True),
                                                (True, False, True, True), (False, False, True, False)])
@pytest.mark.parametrize("rows,blocks", [(1, 1), (50, 5), (592, 148)])
def test_backward(kernels, rows, blocks, post, dh_, dy_, gate_):
    import paper_2003_11666_b200 as p
    g = torch.Generator(device="cuda").manual_seed(rows)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    u, y, dy, dh = (rand(rows, 2048).to(torch.bfloat16) for _ in range(4))
    dy, dh = dy if dy_ else None, dh if dh_ else None
    gate = rand(1, 2048).to(torch.bfloat16) if gate_ else None
    a, b = rand(2048) if post else None, rand(2048) if dh_ else None
    rp, rr = rand(rows).abs() if post else None, rand(rows).abs() if dh_ else None
    out = []
    for wait in (WAIT, 0):
        dx, du = torch.zeros_like(u), torch.zeros_like(u)
        da, db = (torch.zeros(blocks, 2048, device="cuda") if t is not None else None for t in (a, b))
        dg = torch.zeros(1, 2048, device="cuda", dtype=torch.bfloat16) if gate_ and blocks == 1 else None
        torch.cuda.synchronize()
        assert kernels.backward(rows, blocks, *(_at(t) for t in (u, y, dy, dh, gate, a, b, rp, rr, dx, du, dg, db, da)), wait) == 0
        out.append((dx, du, dg, da, db))
    want = [torch.zeros_like(u), torch.zeros_like(u), torch.zeros(1, 2048, device="cuda", dtype=torch.bfloat16) if gate_ else None,
            *(torch.zeros(2048, device="cuda") if t is not None else None for t in (a, b))]
    sc = torch.empty(p.join_scratch_bytes(rows, 2048, rows if gate_ else 0), device="cuda", dtype=torch.uint8)
    p.join_backward(y, u, want[0], want[1], sc, dy=dy, dh=dh, pre_weight=b, post_weight=a, gate=gate, rstd_pre=rr, rstd_post=rp, dpost_weight=want[3],
                    dpre_weight=want[4], dgate=want[2])
    for k, (got, ref, lost) in enumerate(zip(out[0], want, out[1])):
        if got is None:
            continue
        total = got.sum(0) if k > 2 else got                       # of the blocks' parts
        step = 2.0 ** -7 if got.dtype is torch.bfloat16 else 0.0
        # sums of `rows` numbers in another order: rows U of their magnitudes, which are below 2^9 each (products of a few normal numbers)
        assert bool(((total.double() - ref.double()).abs() <= step * ref.double().abs() + (rows + 64) * 2.0 ** -24 * 2.0 ** 9 * max(1, rows) ** 0.5).all()), k
        assert bool(lost.isnan().all()), k
