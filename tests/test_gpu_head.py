"""Log probabilities of hidden states under an output head, and their gradients, on the GPU against float64.
Bounds are derived in tests/blocks_ref.py."""
import pytest
import torch

from tests import blocks_ref as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _p():
    import paper_2003_11666_b200 as p
    return p


def _matrix(a, dtype, pad=0, offset=0):
    """[rows, cols] with a row stride of cols + pad that starts `offset` elements into its buffer."""
    rows, cols = a.shape
    flat = torch.full((offset + rows * (cols + pad) + 32,), 7.0, device="cuda", dtype=dtype)
    view = flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(a)
    return flat, view


def _case(rows, vocab, dim, dtype, pad=0, offset=0, seed=0, ids=torch.int64):
    g = torch.Generator(device="cuda").manual_seed(seed + rows + vocab)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    _, h = _matrix(rand(rows, dim), dtype, pad, offset)
    _, w = _matrix(rand(vocab, dim) * (2.0 / dim ** 0.5), dtype, pad, offset)
    tok = torch.randint(0, vocab, (rows,), generator=g, device="cuda").to(ids)
    if rows > 2:
        tok[1] = -1
    h[0] += (w[tok[0].long()].float() * (9.0 / w[tok[0].long()].float().square().sum())).to(dtype)      # a confident row
    return h, w, tok, rand


def _scratch(h, w, backward=False):
    return torch.full((_p().head_scratch_bytes(h, w, backward),), 0xFF, device="cuda", dtype=torch.uint8)


def _forward(h, w, tok, it, **kw):
    rows = h.shape[0]
    out = [torch.full((rows,), 9.0, device="cuda") for _ in range(3)]
    _p().head_logprob_forward(h, w, _scratch(h, w), tok, out[0] if tok is not None else None, entropy=out[1], lse=out[2], inv_temperature=it, **kw)
    return out


def _within(got, ref, tol):
    d = (got.double() - ref).abs()
    bad = ~(d <= tol)
    assert not bool(bad.any()), (int(bad.sum()), float(d[bad].max()), float(tol.expand_as(d)[bad].min()))


def _check_forward(h, w, tok, it):
    logp, entropy, lse = _forward(h, w, tok, it)
    rl, re, rz, _ = R.head_forward(h, w, tok, it)
    el, ee, ez = R.head_forward_error(h, w, tok, it)
    _within(logp, rl, el)
    _within(entropy, re, ee)
    _within(lse, rz, ez)
    return logp, entropy, lse


def _check_backward(h, w, tok, it, rand, lse, entropy, out_type=None, accumulate=False, pad=0, offset=0, parts=("gl", "ge", "gz")):
    p, rows = _p(), h.shape[0]
    dtype = h.dtype
    gl = -(rand(rows).abs() + 0.1) / rows if "gl" in parts else None
    ge = rand(rows) * 0.05 / rows if "ge" in parts else None
    gz = rand(rows) * 0.01 / rows if "gz" in parts else None
    fh, dh = _matrix(torch.zeros(h.shape), dtype, pad, offset)
    fw, dw = _matrix(rand(*w.shape) * 0.01 / rows, out_type or dtype, pad, offset)
    start = dw.double().clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    p.head_logprob_backward(h, w, _scratch(h, w, True), tok, lse, dh, dw, g_logp=gl, g_entropy=ge, entropy=entropy, g_lse=gz, inv_temperature=it,
                            accumulate=accumulate, status=status)
    args = (h, w, tok, it, lse, entropy, gl, ge, gz)
    _, rh, rw, _ = R.head_backward(*args)
    half = 0 if dtype is torch.float32 else STORE[dtype]
    eh, ew = R.head_backward_error(*args, half, STORE[dtype])
    tiny = {torch.float32: 0, torch.bfloat16: 0, torch.float16: 2.0 ** -25}          # half of float16's smallest number
    _within(dh, rh, eh + tiny[dtype])
    if accumulate:
        rw = rw + start
    if out_type or accumulate:
        ew = ew + STORE[dw.dtype] * rw.abs() + U * (start.abs() + rw.abs())
    _within(dw, rw, ew + tiny[dw.dtype])
    assert int(status) == 0
    dh.fill_(7.0), dw.fill_(7.0)
    assert bool((fh == 7.0).all()) and bool((fw == 7.0).all())                     # nothing beside the rows was written


SIZES = [(1, 1, 1), (1, 2, 8), (3, 7, 5), (1, 500, 64), (128, 257, 72), (129, 1000, 33), (300, 1001, 200), (257, 513, 1001), (64, 20000, 128),
         (700, 2900, 520), (5, 130, 4100), (256, 256, 64)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,vocab,dim", SIZES)
def test_sizes_and_types(rows, vocab, dim, dtype):
    h, w, tok, rand = _case(rows, vocab, dim, dtype)
    for it in (1.0, 0.6):
        _, entropy, lse = _check_forward(h, w, tok, it)
        _check_backward(h, w, tok, it, rand, lse, entropy)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("pad,offset", [(8, 0), (16, 16), (3, 0), (0, 1), (8, 4), (5, 3)])
def test_strides_and_alignment(pad, offset, dtype):
    for rows, vocab, dim in ((200, 700, 96), (7, 300, 61)):
        h, w, tok, rand = _case(rows, vocab, dim, dtype, pad, offset, ids=torch.int32)
        _, entropy, lse = _check_forward(h, w, tok, 1.1)
        _check_backward(h, w, tok, 1.1, rand, lse, entropy, pad=pad, offset=offset, accumulate=True)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("accumulate", [False, True])
def test_float32_gradients_of_the_head(dtype, accumulate):
    for rows, vocab, dim in ((130, 600, 72), (260, 300, 19)):
        h, w, tok, rand = _case(rows, vocab, dim, dtype)
        _, entropy, lse = _forward(h, w, tok, 1.0)
        _check_backward(h, w, tok, 1.0, rand, lse, entropy, out_type=torch.float32, accumulate=accumulate)


# pieces of the vocabulary: d of 8192 rows or more in three planes, of 16384 in one; packed weights of many columns
@pytest.mark.parametrize("rows,vocab,dim,dtype", [(8200, 20011, 24, torch.float32), (17000, 17003, 40, torch.bfloat16), (150, 24001, 4104, torch.float32)])
def test_pieces_of_the_vocabulary(rows, vocab, dim, dtype):
    h, w, tok, rand = _case(rows, vocab, dim, dtype)
    _, entropy, lse = _check_forward(h, w, tok, 0.9)
    _check_backward(h, w, tok, 0.9, rand, lse, entropy)
    _check_backward(h, w, tok, 0.9, rand, lse, entropy, accumulate=True)


@pytest.mark.parametrize("parts", [("gl",), ("ge",), ("gz",), ()])
def test_gradients_of_single_values(parts):
    for rows in (40, 200):
        h, w, tok, rand = _case(rows, 900, 72, torch.bfloat16)
        _, entropy, lse = _forward(h, w, tok, 1.0)
        _check_backward(h, w, tok, 1.0, rand, lse, entropy, parts=parts)


def test_one_gradient_alone_and_none_of_the_values():
    p = _p()
    h, w, tok, rand = _case(150, 800, 64, torch.bfloat16)
    _, entropy, lse = _forward(h, w, tok, 1.0)
    gl = rand(150)
    both = [torch.empty_like(h), torch.empty_like(w)]
    p.head_logprob_backward(h, w, _scratch(h, w, True), tok, lse, *both, g_logp=gl)
    one = torch.empty_like(h)
    p.head_logprob_backward(h, w, _scratch(h, w, True), tok, lse, one, None, g_logp=gl)
    assert torch.equal(one, both[0])
    other = torch.empty_like(w)
    p.head_logprob_backward(h, w, _scratch(h, w, True), tok, lse, None, other, g_logp=gl)
    assert torch.equal(other, both[1])
    alone = torch.empty(150, device="cuda")
    p.head_logprob_forward(h, w, _scratch(h, w), lse=alone)
    assert torch.equal(alone, lse)
    p.head_logprob_forward(h, w, _scratch(h, w))
    # no rows: nothing happens to what is added to, and the rest is cleared
    none, n = h[:0], torch.empty(0, device="cuda")
    p.head_logprob_backward(none, w, _scratch(h, w, True), tok[:0], n, none, other, g_logp=n, accumulate=True)
    assert torch.equal(other, both[1])
    wide = torch.full((800, 70), 3.0, device="cuda")
    p.head_logprob_backward(none, w, _scratch(h, w, True), tok[:0], n, None, wide[:, :64], g_logp=n)
    assert bool((wide[:, :64] == 0).all()) and bool((wide[:, 64:] == 3).all())
    p.head_logprob_forward(none, w, _scratch(h, w), tok[:0], n)


def test_tokens_that_are_none():
    p = _p()
    h, w, tok, rand = _case(6, 500, 64, torch.float16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tok[:] = -1
    logp, entropy, lse = _forward(h, w, tok, 1.0, status=status)
    assert bool((logp == 0).all()) and int(status) == 0
    dh, dw = torch.full_like(h, 3.0), torch.full_like(w, 3.0)
    p.head_logprob_backward(h, w, _scratch(h, w, True), tok, lse, dh, dw, g_logp=rand(6))
    assert bool((dh == 0).all()) and bool((dw == 0).all())
    tok[:] = torch.tensor([0, 500, 3, -2, 499, 2 ** 40], device="cuda")
    logp, *_ = _forward(h, w, tok, 1.0, status=status)
    assert int(status) == 1 and bool((logp[[1, 3, 5]] == 0).all()) and bool((logp[[0, 2, 4]] < 0).all())
    status.zero_()
    p.head_logprob_backward(h, w, _scratch(h, w, True), tok, lse, dh, dw, g_logp=rand(6), status=status)
    assert int(status) == 1 and bool((dh[[1, 3, 5]] == 0).all()) and bool((dh[[0, 2, 4]] != 0).any(1).all())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows", [9, 300])
def test_rows_that_are_not_finite_stay_alone(rows, dtype):
    p = _p()
    h, w, tok, rand = _case(rows, 700, 72, dtype)
    clean, _, _ = _forward(h, w, tok, 1.0)
    h[3, 5], h[6, 0] = float("nan"), float("inf")
    logp, entropy, lse = _forward(h, w, tok, 1.0)
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[[3, 6]] = False
    assert torch.equal(logp[rest], clean[rest]) and bool(torch.isnan(lse[3])) and bool(torch.isnan(entropy[3]))
    assert not bool(torch.isfinite(lse[6]))
    gl = rand(rows)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    p.head_logprob_backward(h, w, _scratch(h, w, True), tok, lse, dh, dw, g_logp=gl)
    assert bool(torch.isnan(dh[3]).all()) and bool(torch.isfinite(dh[rest]).all())
    # a gradient that is not finite stays in its row of dhidden
    h2, w2, tok2, rand = _case(rows, 700, 72, dtype)
    _, _, lse2 = _forward(h2, w2, tok2, 1.0)
    ref = torch.empty_like(h)
    p.head_logprob_backward(h2, w2, _scratch(h2, w2, True), tok2, lse2, ref, dw, g_logp=gl)
    gl = gl.clone()
    gl[2] = float("nan")
    p.head_logprob_backward(h2, w2, _scratch(h2, w2, True), tok2, lse2, dh, dw, g_logp=gl)
    keep = torch.arange(rows, device="cuda") != 2
    assert bool(torch.isnan(dh[2]).any()) and bool(torch.isfinite(dh[keep]).all())
    # their scale may differ by a power of two: what is rounded twice is off by two half steps, of the terms' size
    assert float((dh[keep].double() - ref[keep].double()).norm() / ref[keep].double().norm()) < 4 * STORE[dtype] + 2.0 ** -20


def test_gradients_keep_their_digits_at_any_scale():
    # 1e-30, as behind many layers, and 1e6, as behind a loss scale
    for dtype in TYPES:
        h, w, tok, rand = _case(140, 600, 64, dtype)
        _, entropy, lse = _forward(h, w, tok, 1.0)
        gl = rand(140)
        out = []
        for f in (1.0, 2.0 ** -100, 2.0 ** 20):
            dw = torch.empty(w.shape, device="cuda")
            _p().head_logprob_backward(h, w, _scratch(h, w, True), tok, lse, None, dw, g_logp=gl * f)
            out.append(dw.double() / f)
        assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])


def test_gradient_is_the_difference_quotient():
    p = _p()
    h, w, tok, rand = _case(5, 300, 40, torch.float32)
    tok[1] = 7
    ways = rand(5, 40), rand(300, 40) * 0.1

    def value(hh, ww):
        logp, entropy, lse = _forward(hh, ww, tok, 0.8)
        return float((logp.double() + 0.5 * entropy.double() + 0.25 * lse.double()).sum())
    logp, entropy, lse = _forward(h, w, tok, 0.8)
    one = torch.ones(5, device="cuda")
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    p.head_logprob_backward(h, w, _scratch(h, w, True), tok, lse, dh, dw, g_logp=one, g_entropy=0.5 * one, entropy=entropy, g_lse=0.25 * one, inv_temperature=0.8)
    step = 2.0 ** -7
    for way, grad, at in ((ways[0], dh, lambda s: (h + s * way, w)), (ways[1], dw, lambda s: (h, w + s * way))):
        quotient = (value(*at(step)) - value(*at(-step))) / (2 * step)
        # along the way the logits move by m = |z'| at most; third derivatives of lse and the entropy are below 8 m^3 per row; 15 values of
        # size below 16 are known to 2^-20
        m = 0.8 * float(((way @ w.T).abs() if way is ways[0] else (h @ way.T).abs()).max())
        assert abs(quotient - float((grad.double() * way.double()).sum())) < 5 * 3 * 8 * m ** 3 * step ** 2 / 6 + 15 * 2.0 ** -16 / step


@pytest.mark.parametrize("rows", [1, 64, 400])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_captured_calls_replay_beside_each_other(rows, dtype):
    p = _p()

    def state(seed):
        h, w, tok, rand = _case(rows, 3000, 136, dtype, seed=seed)
        s = dict(h=h, w=w, tok=tok, src=h.clone(), logp=torch.zeros(rows, device="cuda"), lse=torch.zeros(rows, device="cuda"), dh=torch.zeros_like(h),
                 dw=torch.zeros_like(w), gl=rand(rows), f=_scratch(h, w), b=_scratch(h, w, True))
        return s

    def step(s):
        s["h"].copy_(s["src"])
        p.head_logprob_forward(s["h"], s["w"], s["f"], s["tok"], s["logp"], lse=s["lse"])
        p.head_logprob_backward(s["h"], s["w"], s["b"], s["tok"], s["lse"], s["dh"], s["dw"], g_logp=s["gl"])
    names = ("logp", "lse", "dh", "dw")
    eager, captured = [state(k) for k in range(2)], [state(k) for k in range(2)]
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for s, stream in zip(captured, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(s)
        graphs.append(graph)
    for k in range(3):
        for s in eager + captured:
            s["src"].mul_(0.9)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, captured):
            step(a)
            for n in names:
                assert torch.equal(a[n], b[n]), n


def test_calls_follow_the_current_stream():
    p = _p()
    h, w, tok, _ = _case(200, 900, 64, torch.bfloat16)
    ref, *_ = _forward(h, w, tok, 1.0)
    late, out, sc = torch.zeros_like(h), torch.empty(200, device="cuda"), _scratch(h, w)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
        late.copy_(h)
        p.head_logprob_forward(late, w, sc, tok, out)
    stream.synchronize()
    assert torch.equal(ref, out)


def test_offsets_pass_32_bits():
    p = _p()
    vocab, dim = 300_000, 8192                                    # 2.5e9 elements, 4.9 GB
    w = torch.zeros(vocab, dim, device="cuda", dtype=torch.bfloat16)
    w[-1, :64], w[5, :64] = 0.25, -0.25
    h = torch.zeros(3, dim, device="cuda", dtype=torch.bfloat16)
    h[:, :64] = 0.5
    tok = torch.tensor([vocab - 1, 5, 0], device="cuda")
    logp, entropy, lse = _forward(h, w, tok, 1.0)
    z = torch.zeros(vocab, device="cuda", dtype=torch.float64)
    z[-1], z[5] = 8.0, -8.0
    ref = torch.log_softmax(z, 0)
    # sums of 300000 ones in 2^-20
    _within(logp, ref[tok], torch.tensor(2.0 ** -19, device="cuda"))
    dh, dw = torch.empty_like(h), torch.full_like(w, 3.0)
    p.head_logprob_backward(h, w, _scratch(h, w, True), tok, lse, dh, dw, g_logp=torch.ones(3, device="cuda"))
    d = -3 * ref.exp()
    d[tok] += 1
    _within(dw[[0, 5, vocab - 2, vocab - 1], 3], 0.5 * d[[0, 5, vocab - 2, vocab - 1]], 0.5 * (3 * 2.0 ** -8 + 2.0 ** -18) * (3 * ref.exp() + (d > 0))[[0, 5, vocab - 2, vocab - 1]])
    assert bool((dw[:, 64:] == 0).all())


# rows that run without the tensor cores: odd widths at strides of 16 bytes, vocabularies shorter than a block and longer than a round of all of them
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("vocab,dim,pad", [(1, 512, 0), (7, 1021, 3), (9475, 513, 7), (50021, 776, 8), (300, 9000, 0)])
def test_a_few_rows(rows, vocab, dim, pad, dtype):
    h, w, tok, rand = _case(rows, vocab, dim, dtype, pad)
    _check_forward(h, w, tok, 0.8)
    logp, entropy, lse = _forward(h, w, tok, 0.8)
    again = _forward(h, w, tok, 0.8)
    assert all(torch.equal(a, b) for a, b in zip((logp, entropy, lse), again))
    lse_only = torch.full((rows,), 9.0, device="cuda")
    _p().head_logprob_forward(h, w, _scratch(h, w), lse=lse_only, inv_temperature=0.8)
    assert torch.equal(lse_only, lse)
    h[0, dim - 1] = float("nan")
    bad = _forward(h, w, tok, 0.8)
    assert all(bool(b[0].isnan()) and torch.equal(b[1:], a[1:]) for a, b in zip((logp, entropy, lse), bad))


def test_a_float32_scratch_serves_any_rows():
    lib = __import__("paper_2003_11666_b200.binding", fromlist=["load_library"]).load_library()
    for rows, vocab, dim in ((1, 1, 1), (1, 1000, 1), (4, 100, 3), (4, 100000, 64)):
        assert lib.pb_head_scratch_bytes(0, rows, vocab, dim, 1, 0) == lib.pb_head_scratch_bytes(0, rows, vocab, dim, 0, 0)
