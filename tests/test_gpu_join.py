"""Joins of a block to the residual stream, their gradient, and dropout, on the GPU against float64.  Bounds: see
tests/blocks_ref.py; a store rounds by half a step (2^-24, 2^-8, 2^-11 of the value; float16 by 2^-25 at least)."""
import pytest
import torch

from tests import blocks_ref as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {torch.float32: (U, 0.0), torch.bfloat16: (2.0 ** -8, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25)}
TYPES = [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16),
         (torch.float16, torch.float32)]
EPS = 1e-5


def _p():
    import paper_2003_11666_b200 as p
    return p


def _matrix(a, dtype, pad=0, offset=0):
    rows, cols = a.shape
    flat = torch.full((offset + rows * (cols + pad) + 32,), 7.0, device="cuda", dtype=dtype)
    view = flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(a)
    return flat, view


def _within(got, ref, tol, dtype=None):
    rel, ab = STORE[dtype or got.dtype]
    d = (got.double() - ref).abs()
    bad = ~(d <= tol + rel * (ref.abs() + tol) + ab)
    assert not bool(bad.any()), (int(bad.sum()), float(d[bad].max()), float(ref[bad].abs().max()))


def _factor(seed, offset, p, rows, dim):
    return R.keep(seed, offset, p, rows, dim).cuda() if p else None


def _run(rows, dim, types, per=None, post=True, pre=True, p=0.0, pad=0, offset=0, wtype=torch.float32, gtype=None, seed=0, in_place=False):
    pb, (dt, st) = _p(), types
    g = torch.Generator(device="cuda").manual_seed(seed + rows * 7 + dim)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    put = lambda a, t: _matrix(a, t, pad, offset)                 # noqa: E731
    _, x = put(rand(rows, dim) * 2, st)
    _, u = put(rand(rows, dim) * 3, dt)
    gate = put(rand(-(-rows // per), dim), dt)[1] if per else None
    a = (rand(dim).abs() + 0.3).to(wtype) if post else None
    b = (rand(dim).abs() + 0.3).to(wtype) if pre else None
    rs, sd, off = 0.75, 2 ** 63 + seed, 5
    fy, y = put(torch.zeros(rows, dim), st)
    fh, h = put(torch.zeros(rows, dim), dt)
    rp, rr = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    f = _factor(sd, off, p, rows, dim)
    ry, rh, rrp, rrr = R.join_forward(x, u, gate, per, a, b, rs, EPS, f)
    kw = dict(pre_weight=b, post_weight=a, gate=gate, rows_per_gate=per, rstd_post=rp if post else None, rstd_pre=rr if pre else None, residual_scale=rs, p=p,
              seed=sd, offset=off)
    if in_place:
        y, h = x, u.clone()
        fy = fh = None
        u2 = h
    else:
        u2 = u
    pb.join_forward(x, u2, y, h=h if pre else None, eps=EPS, **kw)
    # rstd: a mean of dim squares, 34 U of itself, halved by the root, which costs 2 U
    branch = ry - rs * (x.double() if not in_place else 0) if not in_place else None
    ty = 40 * U * (branch.abs() if branch is not None else ry.abs() + 8) + 2 * U * ry.abs()
    _within(y, ry, ty)
    if post:
        _within(rp, rrp, 20 * U * rrp)
    if pre:
        # the norm's sum moves with y: by less than the largest error's share of a row's length
        move = (ty.square().sum(1) / ry.square().sum(1).clamp(min=1e-30)).sqrt()[:, None]
        _within(rr, rrr, 20 * U * rrr + move[:, 0] * rrr)
        _within(h, rh, rh.abs() * (24 * U + move) + ty * rrr[:, None] * b.double().abs())
    if in_place:
        return
    if not pre:
        assert bool((fh[offset:offset + rows * (dim + pad)].view(rows, dim + pad)[:, :dim] == 0).all())
    y.fill_(7.0), h.fill_(7.0)
    assert bool((fy == 7.0).all()) and bool((fh == 7.0).all())

    # backward, from what the forward left in the stream's type
    y.copy_(ry)
    rp.copy_(rrp) if post else None
    rr.copy_((y.double().square().mean(1) + EPS).rsqrt())
    _, dy = put(rand(rows, dim), st)
    _, dh = put(rand(rows, dim), dt)
    for dy_, dh_ in ((dy, dh if pre else None), (None, dh)) if pre else ((dy, None),):
        fx, dx = put(torch.zeros(rows, dim), st)
        fu, du = put(torch.zeros(rows, dim), dt)
        fg, dg = put(torch.zeros(gate.shape), gtype or dt) if per else (None, None)
        da = torch.empty(dim, device="cuda", dtype=wtype) if post else None
        db = torch.empty(dim, device="cuda", dtype=wtype) if dh_ is not None else None
        scratch = torch.full((pb.join_scratch_bytes(rows, dim, per or 0),), 0xFF, device="cuda", dtype=torch.uint8)
        pb.join_backward(y, u, dx, du, scratch, dy=dy_, dh=dh_, dpre_weight=db, dpost_weight=da, dgate=dg, **kw)
        ref = R.join_backward(y, u, dy_, dh_, gate, per or rows, a, b, rp if post else None, rr, rs, f)
        for got, name in ((dx, "dx"), (du, "du"), (dg, "dgate"), (da, "dpost"), (db, "dpre")):
            if got is not None:
                _within(got, ref[name], ref["e_" + name])
        dx.fill_(7.0), du.fill_(7.0)
        assert bool((fx == 7.0).all()) and bool((fu == 7.0).all())
        if per:
            dg.fill_(7.0)
            assert bool((fg == 7.0).all())


SIZES = [(1, 1), (1, 8), (3, 5), (7, 64), (33, 129), (2, 1000), (65, 1001), (5, 4096), (4, 4104), (3, 8192), (2, 16384), (2, 9999), (300, 24), (1, 16383)]


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("rows,dim", SIZES)
def test_sizes_and_types(rows, dim, types):
    _run(rows, dim, types, per=max(1, rows // 3), p=0.25)
    _run(rows, dim, types)


@pytest.mark.parametrize("pad,offset", [(8, 0), (16, 16), (3, 0), (0, 1), (8, 8), (5, 2)])
@pytest.mark.parametrize("types", TYPES[:3], ids=str)
def test_strides_and_alignment(types, pad, offset):
    for dim in (96, 61):
        _run(20, dim, types, per=6, p=0.1, pad=pad, offset=offset, wtype=types[0])


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("pre", [False, True])
@pytest.mark.parametrize("per", [None, 1, 5, 40, 100])
def test_parts(post, pre, per):
    _run(40, 72, TYPES[2], per=per, post=post, pre=pre, gtype=torch.float32)
    _run(40, 72, TYPES[1], per=per, post=post, pre=pre, p=0.4, wtype=torch.bfloat16)


# gates whose rows are one chunk, several, of several workers; more chunks than workers; a short last gate
@pytest.mark.parametrize("rows,dim,per", [(5000, 512, 5000), (5000, 512, 1700), (3001, 40, 3001), (20000, 16, 3), (4100, 4096, 1000), (70000, 16, 9), (1500, 2056, 1)])
def test_many_rows(rows, dim, per):
    _run(rows, dim, TYPES[1], per=per, p=0.1)
    _run(rows, dim, TYPES[0], per=per)


# rows in the ring: every thread with all its columns, and not; a gate for each row, for some, for all; 1024 threads; two rows in flight, or none
@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("rows,dim,per", [(1500, 1024, 700), (700, 1032, 1), (2000, 528, 3), (640, 4096, 640), (600, 5120, 5), (601, 8192, 300), (600, 8200, 600)])
def test_rows_in_the_ring(rows, dim, per, types):
    _run(rows, dim, types, per=per, p=0.2)
    _run(rows, dim, types, per=None, post=True)


def test_more_gates_of_several_chunks_than_a_grid_has_in_one_direction():
    rows, dim, per = 2_500_000, 16, 36                            # 69445 gates; 33 rows per chunk
    _run(rows, dim, (torch.float32, torch.float32), per=per, post=False, pre=False)


def test_in_place():
    for types in TYPES:
        _run(30, 264, types, per=7, in_place=True)
    pb = _p()
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    y, u, dy, dh, w = rand(30, 264), rand(30, 264), rand(30, 264), rand(30, 264), rand(264)
    rr, rp = (y.square().mean(1) + EPS).rsqrt(), (u.square().mean(1) + EPS).rsqrt()
    scratch = torch.empty(pb.join_scratch_bytes(30, 264), device="cuda", dtype=torch.uint8)
    out = [torch.empty_like(y), torch.empty_like(u)]
    kw = dict(pre_weight=w, post_weight=w, rstd_pre=rr, rstd_post=rp, p=0.3, seed=1)
    pb.join_backward(y, u, *out, scratch, dy=dy, dh=dh, **kw)
    pb.join_backward(y, u, dy, dh, scratch, dy=dy, dh=dh, **kw)
    assert torch.equal(dy, out[0]) and torch.equal(dh, out[1])
    pb.join_backward(y, u, None, out[0], scratch, dy=out[0].clone(), **{**kw, "rstd_pre": None, "pre_weight": None})      # no dx


def test_rows_that_are_not_finite_stay_alone():
    pb = _p()
    for types in TYPES[:3]:
        dt, st = types
        x, u = torch.randn(9, 200, device="cuda").to(st), torch.randn(9, 200, device="cuda").to(dt)
        w = torch.rand(200, device="cuda") + 0.5
        ref = [torch.empty_like(x), torch.empty_like(u)]
        pb.join_forward(x, u, ref[0], h=ref[1], pre_weight=w, post_weight=w)
        u[4, 7], x[6, 0] = float("nan"), float("inf")
        got = [torch.empty_like(x), torch.empty_like(u)]
        pb.join_forward(x, u, got[0], h=got[1], pre_weight=w, post_weight=w)
        rest = torch.tensor([0, 1, 2, 3, 5, 7, 8], device="cuda")
        for a, b in zip(ref, got):
            assert torch.equal(a[rest], b[rest])
        assert bool(torch.isnan(got[0][4]).all()) and bool(torch.isinf(got[0][6, 0])) and bool(torch.isnan(got[1][6, 0]))
    # rows of nothing but zeros: eps alone
    z = torch.zeros(2, 64, device="cuda")
    y, h, rr = torch.empty_like(z), torch.empty_like(z), torch.empty(2, device="cuda")
    pb.join_forward(z, z, y, h=h, pre_weight=w[:64].contiguous(), post_weight=w[:64].contiguous(), rstd_pre=rr, eps=0.25)
    assert bool((h == 0).all()) and bool((rr == 2.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("rows,dim", [(1, 1), (1, 7), (3, 8), (5, 33), (64, 1000), (301, 1001), (7, 100_003)])
def test_dropout(rows, dim, dtype):
    pb = _p()
    for p, seed, offset in ((0.0, 1, 0), (0.1, 2 ** 64 - 3, 2 ** 40), (0.5, -1, 1), (0.998, 12345, 7)):
        for pad, at in ((0, 0), (8, 8), (3, 1)):
            _, x = _matrix(torch.randn(rows, dim, device="cuda"), dtype, pad, at)
            flat, out = _matrix(torch.zeros(rows, dim), dtype, pad, at)
            pb.dropout(x, out, p, seed, offset=offset)
            ref = x.double() * R.keep(seed % 2 ** 64, offset, p, rows, dim).cuda()
            _within(out, ref, U * 2 * ref.abs())
            in_place = x.clone() if not pad else None
            if in_place is not None:
                pb.dropout(in_place, in_place, p, seed, offset=offset)
                assert torch.equal(in_place, out)
            out.fill_(7.0)
            assert bool((flat == 7.0).all())


def test_dropped_elements_are_zero_whatever_they_were():
    pb = _p()
    x = torch.full((4, 512), float("nan"), device="cuda")
    out = torch.empty_like(x)
    pb.dropout(x, out, 0.5, 9)
    f = R.keep(9, 0, 0.5, 4, 512).cuda()
    assert bool((out[f == 0] == 0).all()) and bool(torch.isnan(out[f > 0]).all())


def test_offsets_on_the_device_in_captured_graphs():
    pb = _p()
    x, u, w = torch.randn(6, 96, device="cuda"), torch.randn(6, 96, device="cuda"), torch.rand(96, device="cuda")
    out, y, dx, du = (torch.empty_like(x) for _ in range(4))
    off = torch.zeros(1, dtype=torch.int64, device="cuda")
    scratch = torch.empty(pb.join_scratch_bytes(6, 96), device="cuda", dtype=torch.uint8)

    def step(**kw):
        pb.dropout(x, out, 0.3, 5, **kw)
        pb.join_forward(x, u, y, p=0.3, seed=6, **kw)
        pb.join_backward(None, u, dx, du, scratch, dy=x, p=0.3, seed=6, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(offset=77, dev_offset=off)
        off.add_(1)
    seen = []
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, y, dx, du)]
        step(offset=k)
        for a, b in zip(got, (out, y, dx, du)):
            assert torch.equal(a, b)
        seen.append(got[0])
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


def test_gradient_is_the_difference_quotient():
    pb = _p()
    g = torch.Generator(device="cuda").manual_seed(8)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    rows, dim, per = 6, 40, 3
    x, u, gate, a, b = rand(rows, dim), rand(rows, dim), rand(2, dim), rand(dim), rand(dim)
    cy, ch = rand(rows, dim), rand(rows, dim)
    kw = dict(rows_per_gate=per, residual_scale=0.8, p=0.3, seed=4, offset=2)

    def value(x, u, gate, a, b):
        y, h = torch.empty_like(x), torch.empty_like(x)
        rp, rr = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        pb.join_forward(x, u, y, h=h, pre_weight=b, post_weight=a, gate=gate, rstd_pre=rr, rstd_post=rp, eps=EPS, **kw)
        return float((y.double() * cy.double() + h.double() * ch.double()).sum()), y, rp, rr
    _, y, rp, rr = value(x, u, gate, a, b)
    out = [torch.empty_like(t) for t in (x, u, gate, a, b)]
    scratch = torch.empty(pb.join_scratch_bytes(rows, dim, per), device="cuda", dtype=torch.uint8)
    pb.join_backward(y, u, out[0], out[1], scratch, dy=cy, dh=ch, pre_weight=b, post_weight=a, gate=gate, rstd_pre=rr, rstd_post=rp, dgate=out[2],
                     dpost_weight=out[3], dpre_weight=out[4], **kw)
    step = 2.0 ** -8
    for k in range(5):
        at = [x, u, gate, a, b]
        way = rand(*at[k].shape)
        way /= way.norm()                                         # so that derivatives along it are of the size of the function's own
        values = []
        for s in (step, -step):
            moved = list(at)
            moved[k] = at[k] + s * way
            values.append(value(*moved)[0])
        quotient, slope = (values[0] - values[1]) / (2 * step), float((out[k].double() * way.double()).sum())
        # 480 terms of size below 10, each known to 2^-20, over 2 steps; a third derivative of 1000 at most
        assert abs(quotient - slope) < 480 ** 0.5 * 10 * 2.0 ** -20 / step + 1000 * step ** 2 / 6, (k, quotient, slope)


def test_offsets_pass_32_bits():
    pb = _p()
    rows, dim = 140_000, 16384                                    # 2.3e9 elements, 4.6 GB
    x = torch.zeros(rows, dim, device="cuda", dtype=torch.bfloat16)
    x[-1], x[0] = 2.0, 1.0
    pb.dropout(x, x, 0.5, 3, offset=1)
    base = rows * dim - 4096
    f = _last_factors(3, 1, base, 4096)
    assert torch.equal(x.view(-1)[base:].double().cpu(), 2.0 * f)
    u = torch.zeros(1, dim, device="cuda", dtype=torch.bfloat16).expand(rows, dim).contiguous()
    u[-1] = 1.0
    y = x
    pb.join_forward(x, u, y, p=0.5, seed=3, offset=1)
    assert torch.equal(y.view(-1)[base:].double().cpu(), 4.0 * (f > 0) + f)


def _last_factors(seed, offset, first, n):
    """Factors of elements first .. first + n of a call, in Python's whole numbers."""
    m, gamma = (1 << 64) - 1, 0x9E3779B97F4A7C15

    def hashed(base, counter):
        z = (base + (counter + 1) * gamma) & m
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & m
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & m
        return z ^ (z >> 31)
    base = hashed(seed, offset)
    quads = [hashed(base, q) for q in range(first // 4, (first + n) // 4)]
    return torch.tensor([2.0 if (q >> (16 * k)) & 0xFFFF >= 32768 else 0.0 for q in quads for k in range(4)], dtype=torch.float64)


def test_no_rows():
    pb = _p()
    e = lambda *n: torch.empty(*n, device="cuda")                 # noqa: E731
    w, none, no_row = torch.ones(64, device="cuda"), e(0, 64), e(0)
    scratch = torch.empty(pb.join_scratch_bytes(0, 64, 3), device="cuda", dtype=torch.uint8)
    pb.dropout(none, none, 0.5, 1)
    pb.join_forward(none, none, none.clone(), h=none.clone(), pre_weight=w, post_weight=w, gate=none, rows_per_gate=3, rstd_pre=no_row, rstd_post=no_row)
    d = [torch.full((64,), 3.0, device="cuda") for _ in range(2)]
    pb.join_backward(none, none, none.clone(), none.clone(), scratch, dy=none, dh=none, pre_weight=w, post_weight=w, gate=none, rows_per_gate=3, rstd_pre=no_row,
                     rstd_post=no_row, dpre_weight=d[0], dpost_weight=d[1], dgate=none.clone())
    assert not d[0].any() and not d[1].any()                       # sums over nothing


def test_calls_follow_the_current_stream():
    pb = _p()
    x, u, w = torch.randn(1200, 512, device="cuda"), torch.randn(1200, 512, device="cuda"), torch.rand(512, device="cuda")
    scratch = torch.empty(pb.join_scratch_bytes(1200, 512), device="cuda", dtype=torch.uint8)

    def run(x, out):
        pb.dropout(x, out[0], 0.2, 3)
        pb.join_forward(out[0], u, out[1], h=out[2], pre_weight=w, post_weight=w, rstd_pre=out[3], rstd_post=out[4])
        pb.join_backward(out[1], u, out[5], out[6], scratch, dh=out[2], pre_weight=w, post_weight=w, rstd_pre=out[3], rstd_post=out[4], dpre_weight=out[7],
                         dpost_weight=out[8])
    new = lambda: [torch.zeros_like(x) for _ in range(3)] + [torch.zeros(1200, device="cuda") for _ in range(2)] + [torch.zeros_like(x) for _ in range(2)] + \
        [torch.zeros(512, device="cuda") for _ in range(2)]                    # noqa: E731
    ref, got, late = new(), new(), torch.zeros_like(x)
    run(x, ref)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
        late.copy_(x)
        run(late, got)
    stream.synchronize()
    for a, b in zip(ref, got):
        assert torch.equal(a, b)
