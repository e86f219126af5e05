"""Joins whose rows come through the ring in shared memory: each part alone, rows with gaps between them, results in place of the inputs."""
import pytest
import torch

from tests.test_gpu_join import TYPES, _run

pytestmark = pytest.mark.gpu

# 3000 x 1024: 64 threads to a row in the forward, 128 in the gradient; 600 x 4104: columns that the last threads do not have; 700 x 8192: 1024 threads in the gradient
SIZES = [(3000, 1024), (600, 4104), (700, 8192)]


@pytest.mark.parametrize("rows,dim", SIZES)
@pytest.mark.parametrize("post,pre,per", [(True, False, None), (True, False, 100), (False, True, 300), (False, False, 7), (False, True, None), (False, False, None)])
def test_parts(rows, dim, post, pre, per):
    _run(rows, dim, TYPES[1], per=per, post=post, pre=pre, p=0.2)
    _run(rows, dim, TYPES[2], per=per, post=post, pre=pre, gtype=torch.float32)


@pytest.mark.parametrize("rows,dim", SIZES)
@pytest.mark.parametrize("types", TYPES[:3], ids=str)
def test_strides(rows, dim, types):
    _run(rows, dim, types, per=500, p=0.1, pad=8, offset=16, wtype=types[0])
    _run(rows, dim, types, pad=24, offset=8, wtype=types[0])


@pytest.mark.parametrize("rows,dim", SIZES)
@pytest.mark.parametrize("types", TYPES[:3], ids=str)
def test_in_place(rows, dim, types):
    import paper_2003_11666_b200 as p
    dt, st = types
    g = torch.Generator(device="cuda").manual_seed(dim)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    x, u, gate, w = rand(rows, dim).to(st), rand(rows, dim).to(dt), rand(3, dim).to(dt), rand(dim)
    for kw in (dict(post_weight=w), dict(post_weight=w, gate=gate, rows_per_gate=-(-rows // 3), p=0.3, seed=2)):
        y, h = torch.empty_like(x), torch.empty_like(u)
        p.join_forward(x, u, y, h=h, pre_weight=w, **kw)
        a, b = x.clone(), u.clone()
        p.join_forward(a, b, a, h=b, pre_weight=w, **kw)
        assert torch.equal(a, y) and torch.equal(b, h)
        kw.update(rstd_pre=rand(rows).abs(), rstd_post=rand(rows).abs(), pre_weight=w)
        scratch = torch.empty(p.join_scratch_bytes(rows, dim, kw.get("rows_per_gate", 0)), device="cuda", dtype=torch.uint8)
        dy, dh, dx, du = rand(rows, dim).to(st), rand(rows, dim).to(dt), torch.empty_like(x), torch.empty_like(u)
        p.join_backward(y, u, dx, du, scratch, dy=dy, dh=dh, **kw)
        p.join_backward(y, u, dy, dh, scratch, dy=dy, dh=dh, **kw)
        assert torch.equal(dy, dx) and torch.equal(dh, du)
