"""Token operators and the AdamW step on the GPU against the float64 oracle.

Tolerances: a value rounded to a type is off by at most half a step, eps_t / 2 of itself
(2^-24 float32, 2^-8 bfloat16, 2^-11 float16; float16 also half of its smallest step, 2^-25);
a sum of n float32 terms by n 2^-24 of the sum of magnitudes; other terms beside their use.
"""
import numpy as np
import pytest

from oracle import tokens as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = ["float32", "bfloat16", "float16"]


def _torch():
    import torch
    import paper_2003_11666_b200 as p
    return torch, p


def _half(dtype):
    """(relative, absolute) rounding of one store in `dtype`."""
    return {"float32": (U, 0.0), "bfloat16": (2.0 ** -8, 2.0 ** -134), "float16": (2.0 ** -11, 2.0 ** -25)}[str(dtype).replace("torch.", "")]


def _matrix(torch, a, dtype, ld=None, offset=0, fill=7.0):
    """A [rows, cols] view with row stride ld that starts `offset` elements into its buffer."""
    rows, cols = a.shape
    ld = cols if ld is None else ld
    flat = torch.full((offset + rows * ld + 16,), fill, device="cuda", dtype=getattr(torch, dtype))
    view = flat[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(torch.from_numpy(np.asarray(a)))
    return flat, view


def _np(t):
    return t.double().cpu().numpy()


def _close(got, ref, tol):
    got, ref, tol = np.broadcast_arrays(got, ref, tol)
    fin = np.isfinite(ref)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(ref))
    np.testing.assert_array_equal(got[~fin & ~np.isnan(ref)], ref[~fin & ~np.isnan(ref)])
    bad = np.abs(got[fin] - ref[fin]) > tol[fin]
    assert not bad.any(), (int(bad.sum()), np.abs(got[fin] - ref[fin]).max(), got[fin][bad][:4], ref[fin][bad][:4], tol[fin][bad][:4])


# ---------------------------------------------------------------- embedding
EMBED = [(1, 1, 1), (1, 5, 3), (7, 11, 8), (33, 100, 129), (300, 1000, 1024), (64, 50, 2056), (5, 9, 8200)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("id_type", ["int32", "int64"])
@pytest.mark.parametrize("n,vocab,dim", EMBED)
def test_embed_forward(n, vocab, dim, id_type, dtype):
    torch, p = _torch()
    rng = np.random.default_rng(n + dim)
    for ld, offset, ld_out, off_out in ((dim, 0, dim, 0), (dim + 8, 8, dim + 16, 0), (dim + 3, 1, dim + 5, 2)):
        _, table = _matrix(torch, rng.normal(size=(vocab, dim)), dtype, ld, offset)
        ids = rng.integers(0, vocab, n)
        if n > 3:
            ids[2] = -1
        flat, out = _matrix(torch, np.zeros((n, dim)), dtype, ld_out, off_out)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        p.embed_forward(table, torch.tensor(ids, dtype=getattr(torch, id_type), device="cuda"), out, scale=1.7, status=status)
        ref = O.embed_forward(_np(table), ids, float(np.float32(1.7)))
        rel, ab = _half(dtype)
        _close(_np(out), ref, (rel + 2 * U) * np.abs(ref) + ab)
        out.fill_(7.0)
        assert (flat == 7.0).all() and int(status) == 0            # nothing beside the rows was written


def test_embed_reports_ids_out_of_range():
    torch, p = _torch()
    table = torch.ones(4, 6, device="cuda")
    out = torch.full((5, 6), 3.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ids = torch.tensor([0, 4, -1, 3, -7], device="cuda")
    p.embed_forward(table, ids, out, status=status)
    assert int(status) == 1 and out[[1, 2, 4]].abs().max() == 0 and (out[[0, 3]] == 1).all()
    status.zero_()
    scratch = torch.empty(p.embed_scratch_bytes(5, 4, 6), dtype=torch.uint8, device="cuda")
    d = torch.full((4, 6), 3.0, device="cuda")
    p.embed_backward(torch.ones(5, 6, device="cuda"), ids, d, scratch, status=status)
    assert int(status) == 1 and (d[[0, 3]] == 1).all() and d[1:3].abs().max() == 0
    p.embed_backward(torch.ones(5, 6, device="cuda"), ids, d, scratch)      # without a status word
    p.embed_forward(table, ids, out)


def _embed_ids(kind, n, vocab, rng):
    if kind == "uniform":
        return rng.integers(0, vocab, n)
    if kind == "same":
        return np.full(n, vocab // 2)
    if kind == "frequent":                                        # a few long runs, many short ones, padding
        ids = (vocab * rng.random(n) ** 3).astype(np.int64)
        ids[rng.random(n) < 0.3] = vocab - 1
        ids[rng.random(n) < 0.1] = -1
        return ids
    if kind == "none":
        return np.full(n, -1)
    return np.arange(n) % vocab


def _embed_backward(torch, p, n, vocab, dim, dtype, gtype, id_type, kind, accumulate, pad=-1, ld=None, ld_dout=None, offset=0, stream=0):
    rng = np.random.default_rng(n * 7 + dim)
    ids = _embed_ids(kind, n, vocab, rng)
    _, dout = _matrix(torch, rng.normal(size=(n, dim)), dtype, ld_dout, offset)
    flat, d = _matrix(torch, rng.normal(size=(vocab, dim)), gtype, ld, offset)
    start = _np(d)
    scratch = torch.full((p.embed_scratch_bytes(n, vocab, dim),), 0xA5, dtype=torch.uint8, device="cuda")
    dev_ids = torch.tensor(ids, dtype=getattr(torch, id_type), device="cuda")
    torch.cuda.synchronize()
    p.embed_backward(dout, dev_ids, d, scratch, scale=1.7, padding_idx=pad, accumulate=accumulate, stream=stream)
    torch.cuda.synchronize()
    x, s = _np(dout), float(np.float32(1.7))
    ref, mag, count = start.copy() if accumulate else np.zeros((vocab, dim)), np.zeros((vocab, dim)), np.zeros(vocab)
    keep = (ids >= 0) & (ids != pad)
    np.add.at(ref, ids[keep], s * x[keep])
    np.add.at(mag, ids[keep], s * np.abs(x[keep]))
    np.add.at(count, ids[keep], 1)
    rel, ab = _half(gtype)
    tol = (count[:, None] + 2) * U * mag + (rel + 2 * U) * np.abs(ref) + 2 * U * np.abs(start) * accumulate + ab
    got = _np(d)
    untouched = count == 0
    np.testing.assert_array_equal(got[untouched], start[untouched] if accumulate else 0.0)
    _close(got, ref, tol)
    d.fill_(7.0)
    assert (flat == 7.0).all()
    return got


@pytest.mark.parametrize("dtype,gtype", [("float32", "float32"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float16", "float16"),
                                         ("float16", "float32")])
@pytest.mark.parametrize("n,vocab,dim,kind", [(1, 1, 1, "uniform"), (1, 700, 40, "uniform"), (40, 11, 8, "uniform"), (1000, 37, 129, "frequent"),
                                              (2047, 5000, 136, "frequent"), (3001, 64, 520, "same"), (700, 300, 2056, "order"), (5, 9, 8200, "none")])
def test_embed_backward(n, vocab, dim, kind, dtype, gtype):
    torch, p = _torch()
    for accumulate in (False, True):
        _embed_backward(torch, p, n, vocab, dim, dtype, gtype, "int64" if n % 2 else "int32", kind, accumulate)
    _embed_backward(torch, p, n, vocab, dim, dtype, gtype, "int32", kind, True, pad=vocab // 2, ld=dim + 3, ld_dout=dim + 5, offset=1)


@pytest.mark.parametrize("n,vocab,dim,kind", [(20000, 70000, 16, "frequent"), (65536, 131072, 8, "frequent"), (70001, 3, 33, "uniform"),
                                              (30000, 1, 24, "same"), (9000, 200000, 64, "order"), (4097, 4097, 40, "uniform")])
def test_embed_backward_of_many_tokens(n, vocab, dim, kind):
    torch, p = _torch()
    a = _embed_backward(torch, p, n, vocab, dim, "bfloat16", "float32", "int64", kind, False)
    b = _embed_backward(torch, p, n, vocab, dim, "bfloat16", "float32", "int32", kind, False)
    np.testing.assert_array_equal(a, b)                            # the order of the sums depends on the ids alone
    _embed_backward(torch, p, n, vocab, dim, "float32", "float32", "int32", kind, True, pad=vocab - 1)


@pytest.mark.parametrize("n", [50, 2048, 2049, 7000])
@pytest.mark.parametrize("dim,ld", [(64, 64), (64, 67), (33, 40)])
def test_embed_backward_clears_the_padding_row(n, dim, ld):
    torch, p = _torch()
    for kind, pad in (("frequent", 299), ("same", 150), ("uniform", 0)):
        _embed_backward(torch, p, n, 300, dim, "bfloat16", "bfloat16", "int64", kind, False, pad=pad, ld=ld)


@pytest.mark.parametrize("dtype,gtype", [("bfloat16", "float32"), ("float32", "float32"), ("float16", "float16")])
def test_embed_backward_of_wide_rows_and_long_runs(dtype, gtype):
    # runs over many stretches, in several slabs of columns
    torch, p = _torch()
    for kind in ("frequent", "same", "uniform"):
        _embed_backward(torch, p, 5000, 6, 4104, dtype, gtype, "int32", kind, kind == "uniform")
    _embed_backward(torch, p, 4500, 3, 2051, dtype, gtype, "int32", "frequent", True)


def test_embed_backward_of_no_tokens_clears_the_table():
    torch, p = _torch()
    d = torch.ones(10, 12, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    scratch = torch.empty(p.embed_scratch_bytes(0, 10, 12), dtype=torch.uint8, device="cuda")
    p.embed_backward(torch.empty(0, 12, device="cuda"), none, d, scratch, accumulate=True)
    assert (d == 1).all()
    p.embed_backward(torch.empty(0, 12, device="cuda"), none, d, scratch)
    assert (d == 0).all()


def test_embed_gradient_is_the_difference_quotient():
    torch, p = _torch()
    rng = np.random.default_rng(3)
    table, ids, dout, way = rng.normal(size=(9, 5)), rng.integers(0, 9, 30), rng.normal(size=(30, 5)), rng.normal(size=(9, 5))
    d = torch.empty(9, 5, device="cuda")
    scratch = torch.empty(p.embed_scratch_bytes(30, 9, 5), dtype=torch.uint8, device="cuda")
    dev_ids = torch.tensor(ids, device="cuda")
    p.embed_backward(torch.tensor(dout, device="cuda", dtype=torch.float32), dev_ids, d, scratch, scale=0.5)
    value = []
    for h in (0.5, -0.5):                                          # linear: any step will do
        out = torch.empty(30, 5, device="cuda")
        p.embed_forward(torch.tensor(table + h * way, device="cuda", dtype=torch.float32), dev_ids, out, scale=0.5)
        value.append((_np(out) * dout).sum())
    # 150 products, each off by a few roundings of numbers of order 1 to 10
    assert abs((value[0] - value[1]) - (_np(d) * way).sum()) < 150 * 40 * U


# ---------------------------------------------------------------- log probabilities
def _logits(rng, rows, vocab, kind):
    x = rng.normal(size=(rows, vocab)) * 2.5
    if kind == "ties":
        x = np.round(x)
    elif kind == "confident":
        x[np.arange(rows), rng.integers(0, vocab, rows)] += 14.0
    elif kind == "masked":
        x[rng.random((rows, vocab)) < 0.4] = -np.inf
        x[0] = -np.inf                                            # nothing left
        if rows > 2:
            x[1] = -np.inf
            x[1, vocab // 2] = 0.25                               # one token left
    elif kind == "constant":
        x[:] = 0.5
    elif kind == "rising":
        x[:] = np.arange(vocab) / 16.0
    elif kind == "falling":
        x[:] = -np.arange(vocab) / 16.0
    elif kind == "far":
        x = x + 1000.0
    return x


def _logprob_tolerance(x, it, dtype_rows):
    """Worst-case errors of the row values from float32 evaluation of exp(it (x - max)) and sums of them."""
    with np.errstate(invalid="ignore"):
        d = (x - x.max(1, keepdims=True)) * it
    d = np.where(np.isfinite(d), d, -np.inf)
    e = np.exp(d)
    ad = np.where(e > 0, -d, 0.0)
    rest = np.maximum(e.sum(1) - 1.0, 0.0)
    z = 1.0 + rest
    # difference, product and the factor's own rounding: 3 U |d| in the exponent; exp itself and its
    # result 2^-22; sums in chains of at most vocab / 256 + 64 additions
    chain = (x.shape[1] / 256 + 64) * U
    err_e = e * (3 * U * ad + 2.0 ** -22 + chain)
    # exp of anything below -87 is lost (denormal or zero): e^-87 each at most
    err_e = err_e + np.exp(-87.0) * (d > -np.inf)
    err_rest = np.where(d < 0, err_e, 0.0).sum(1)
    err_moment = (np.where(d < 0, err_e, 0.0) * ad + e * ad * (3 * U + chain)).sum(1)
    moment = (e * ad).sum(1)
    return err_rest / z, err_rest / z + err_moment / z + moment / z * (err_rest / z + 4 * U)


def _logprob_case(rows, vocab, dtype, kind, it, k, id_type="int32", ld=None, offset=0, seed=0):
    torch, p = _torch()
    rng = np.random.default_rng(rows * 31 + vocab + seed)
    flat, x = _matrix(torch, _logits(rng, rows, vocab, kind), dtype, ld, offset)
    tok = rng.integers(0, vocab, rows)
    if rows > 4:
        tok[3] = -1
    f = lambda *n: torch.full(n, 9.0, device="cuda")              # noqa: E731
    logp, entropy, lse, top, ids = f(rows), f(rows), f(rows), f(rows, k), torch.full((rows, k), 9, dtype=torch.int32, device="cuda")
    before = flat.clone()
    dev_tok = torch.tensor(tok, dtype=getattr(torch, id_type), device="cuda")
    p.logprob_forward(x, dev_tok, logp, entropy=entropy, lse=lse, top_logp=top if k else None, top_ids=ids if k else None, inv_temperature=it)
    assert torch.equal(flat, before)
    xs = _np(x)
    rl, re, rz, rt, ri = O.logprob_forward(xs, tok, it, k)
    tz, te = _logprob_tolerance(xs, it, rows)
    _close(_np(logp), rl, tz + 2 * U * np.abs(rl))
    _close(_np(entropy), re, te + 2 * U * np.abs(re))
    _close(_np(lse), rz, tz + 2 * U * np.abs(rz))
    np.testing.assert_array_equal(ids.cpu().numpy(), ri)
    _close(_np(top), rt, tz[:, None] + 2 * U * np.abs(rt))
    return x, dev_tok, tok, rz, re, lse, entropy


def _logprob_gradient(torch, p, x, dev_tok, tok, it, dtype, in_place, ld=None, offset=0, which="all"):
    rows, vocab = x.shape
    rng = np.random.default_rng(vocab)
    xs = _np(x)
    _, entropy, lse, _, _ = O.logprob_forward(xs, tok, it)
    gl, gh, gz = (rng.normal(size=rows).astype(np.float32) for _ in range(3))
    if which == "logp":
        gh[:] = gz[:] = 0
    lse32, ent32 = lse.astype(np.float32), entropy.astype(np.float32)
    ref = O.logprob_backward(xs, tok, it, lse32, ent32, gl, gh, gz)
    if in_place:
        d, flat = x, None
    else:
        flat, d = _matrix(torch, np.zeros(x.shape), dtype, ld, offset)
    dev = lambda a: torch.tensor(a, device="cuda")                # noqa: E731
    p.logprob_backward(x, dev_tok, dev(lse32), d, g_logp=dev(gl), g_entropy=None if which == "logp" else dev(gh),
                       entropy=None if which == "logp" else dev(ent32), g_lse=None if which == "logp" else dev(gz), inv_temperature=it)
    with np.errstate(invalid="ignore", over="ignore"):
        lp = xs * it - lse32[:, None].astype(np.float64)
        pr = np.exp(lp)
        live = pr > 0
        # exponent: the factor's rounding and the subtraction's; exp 2^-22
        err_lp = U * (np.abs(xs * it) + 2 * np.abs(lp))
        err_p = np.where(live, pr * (err_lp + 2.0 ** -22), 0.0) + 2.0 ** -126
        absl = np.where(live, np.abs(lp), 0.0) + np.abs(ent32[:, None])
        a, h, z = (np.abs(v).astype(np.float64)[:, None] for v in (gl, gh, gz))
        tol = (a + z) * (err_p + 4 * U * pr) + h * (err_p * absl + pr * np.where(live, err_lp, 0.0) + 6 * U * pr * absl)
        hot = np.arange(vocab)[None] == tok[:, None]
        tol = tol + np.where(hot & np.isfinite(ref), 4 * U * a * np.abs(np.where(live, np.expm1(lp), 1.0)) + 2.0 ** -126, 0.0)
    rel, ab = _half(dtype)
    tol = it * tol + (rel + 2 * U) * np.abs(ref) + ab
    _close(_np(d), ref, np.where(np.isfinite(tol), tol, 0.0))
    if flat is not None:
        d.fill_(7.0)
        assert (flat == 7.0).all()


VOCABS = [1, 2, 7, 8, 31, 33, 255, 256, 257, 300, 1023, 4099, 20011]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_logprob_values_and_gradient(vocab, dtype):
    torch, p = _torch()
    k = min(vocab, 5)
    for rows, it, ld, offset in ((1, 1.0, None, 0), (6, 0.7, vocab + 8 - vocab % 8, 8), (5, 1.6, vocab + 3, 1)):
        x, dev_tok, tok, *_ = _logprob_case(rows, vocab, dtype, "normal", it, k, "int64" if rows > 1 else "int32", ld, offset)
        _logprob_gradient(torch, p, x, dev_tok, tok, it, dtype, False, ld, offset)
        _logprob_gradient(torch, p, x, dev_tok, tok, it, dtype, False, vocab + 5, 3, which="logp")
        _logprob_gradient(torch, p, x, dev_tok, tok, it, dtype, True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["ties", "confident", "masked", "constant", "rising", "falling", "far"])
@pytest.mark.parametrize("vocab,k", [(40, 32), (500, 20), (33001, 32), (2048, 1)])
def test_logprob_rows_of_every_kind(kind, vocab, k, dtype):
    torch, p = _torch()
    x, dev_tok, tok, *_ = _logprob_case(6, vocab, dtype, kind, 1.25, k, seed=5)
    _logprob_gradient(torch, p, x, dev_tok, tok, 1.25, dtype, False)


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 131075, "bfloat16"), (2, 131072, "float32"), (3, 262144, "float16"), (40, 9001, "bfloat16"),
                                              (150, 5003, "float32"), (400, 2500, "bfloat16"), (1200, 600, "float16"), (2, 1100003, "bfloat16")])
def test_logprob_row_counts(rows, vocab, dtype):
    torch, p = _torch()
    for k in (0, 20):
        x, dev_tok, tok, *_ = _logprob_case(rows, vocab, dtype, "ties", 1.0, k, seed=k)
    _logprob_gradient(torch, p, x, dev_tok, tok, 1.0, dtype, False)


def test_logprob_of_more_rows_than_a_grid_has_in_one_direction():
    torch, p = _torch()
    x, dev_tok, tok, *_ = _logprob_case(66000, 5, "bfloat16", "normal", 1.0, 2)
    _logprob_gradient(torch, p, x, dev_tok, tok, 1.0, "bfloat16", False)


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 131075, "bfloat16"), (3, 40000, "float32"), (20, 50001, "float16")])
def test_logprob_captured_and_replayed(rows, vocab, dtype):
    # rows split over clusters, on logits that change between the replays
    torch, p = _torch()
    k, stream = 20, torch.cuda.Stream()
    x = torch.randn(rows, vocab, device="cuda").to(getattr(torch, dtype))
    tok = torch.randint(0, vocab, (rows,), device="cuda")
    f = lambda *n: torch.empty(*n, device="cuda")                 # noqa: E731
    out = [f(rows), f(rows), f(rows), f(rows, k), torch.empty(rows, k, dtype=torch.int32, device="cuda")]

    def call(s):
        p.logprob_forward(x, tok, out[0], entropy=out[1], lse=out[2], top_logp=out[3], top_ids=out[4], stream=s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(stream.cuda_stream)
    for _ in range(3):
        x.copy_(torch.randn(rows, vocab, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        call(0)
        for a, b in zip(got, out):
            assert torch.equal(a, b)
        order = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(got[4].long(), order)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [3, 300, 40000])
def test_logprob_rows_that_are_not_finite(vocab, dtype):
    torch, p = _torch()
    rng = np.random.default_rng(1)
    a = rng.normal(size=(7, vocab))
    a[0, vocab - 1] = np.nan
    a[1, 0] = np.inf
    a[2] = -np.inf
    a[2, 1] = np.nan
    a[3] = np.nan
    a[4, vocab // 2:] = -np.inf
    lowest = float(torch.finfo(getattr(torch, dtype)).min)
    a[5] = lowest                                                 # a mask of the type's lowest value everywhere
    a[6] = lowest
    a[6, 2] = 1.0
    _, x = _matrix(torch, a, dtype)
    tok = np.array([0, 0, 0, 2, 0, 1, 2])
    k = 3
    f = lambda *n: torch.full(n, 9.0, device="cuda")              # noqa: E731
    logp, entropy, lse, top, ids = f(7), f(7), f(7), f(7, k), torch.full((7, k), 9, dtype=torch.int32, device="cuda")
    dev_tok = torch.tensor(tok, device="cuda")
    p.logprob_forward(x, dev_tok, logp, entropy=entropy, lse=lse, top_logp=top, top_ids=ids)
    rl, re, rz, rt, ri = O.logprob_forward(_np(x), tok, 1.0, k)
    np.testing.assert_array_equal(ids.cpu().numpy(), ri)
    for got, ref in ((logp, rl), (entropy, re), (lse, rz), (top, rt)):
        _close(_np(got), ref, 2e-4 * np.maximum(1.0, np.abs(ref)) if vocab > 1000 else 2e-6 * np.maximum(1.0, np.abs(ref)))
    d = torch.empty_like(x)
    p.logprob_backward(x, dev_tok, lse, d, g_logp=f(7))
    got = _np(d)
    assert np.isnan(got[[0, 1, 2, 3]]).any(1).all() and np.isfinite(got[[4, 5, 6]]).all()
    assert (got[4, vocab // 2:] == 0).all()
    x.fill_(-float("inf"))
    p.logprob_forward(x, dev_tok, logp, lse=lse, entropy=entropy)
    p.logprob_backward(x, dev_tok, lse, d, g_logp=f(7), g_entropy=f(7), entropy=entropy, g_lse=f(7))
    assert (d == 0).all()


def test_logprob_optional_parts_and_bad_tokens():
    torch, p = _torch()
    x = torch.randn(5, 1000, device="cuda")
    lse, ids, top = torch.empty(5, device="cuda"), torch.empty(5, 4, dtype=torch.int32, device="cuda"), torch.empty(5, 4, device="cuda")
    p.logprob_forward(x, top_logp=top, top_ids=ids)               # alternatives alone
    assert torch.equal(ids.long(), x.topk(4, 1).indices)
    p.logprob_forward(x, lse=lse)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    logp = torch.empty(5, device="cuda")
    p.logprob_forward(x, torch.tensor([0, 1, 2, 1000, -1], device="cuda"), logp, status=status)
    assert int(status) == 1 and (logp[3:] == 0).all() and (logp[:3] < 0).all()
    status.zero_()
    d = torch.empty_like(x)
    g = torch.ones(5, device="cuda")
    p.logprob_backward(x, torch.tensor([0, 1, 2, -2, -1], device="cuda"), lse, d, g_logp=g, status=status)
    assert int(status) == 1 and (d[3:] == 0).all()
    p.logprob_backward(x, None, lse, d, g_lse=g)
    # softmax: each term off by 2^-21 or so of itself
    assert torch.allclose(d.double(), torch.softmax(x.double(), 1), rtol=2.0 ** -19, atol=0)
    assert torch.allclose(d.sum(1), g, atol=1e-5)


def test_logprob_gradient_is_the_difference_quotient():
    torch, p = _torch()
    rng = np.random.default_rng(9)
    x, tok, way = rng.normal(size=(3, 50)), np.array([1, 49, 7]), rng.normal(size=(3, 50))
    dev = lambda a: torch.tensor(a, device="cuda", dtype=torch.float32)      # noqa: E731
    dev_tok = torch.tensor(tok, device="cuda")
    logp, entropy, lse, d = (torch.empty(3, device="cuda") for _ in range(3)), None, None, None
    logp, entropy, lse = logp
    d = torch.empty(3, 50, device="cuda")
    p.logprob_forward(dev(x), dev_tok, logp, entropy=entropy, lse=lse)
    one = torch.ones(3, device="cuda")
    p.logprob_backward(dev(x), dev_tok, lse, d, g_logp=one, g_entropy=one, entropy=entropy, g_lse=one)
    values, h = [], 1e-2
    for s in (h, -h):
        p.logprob_forward(dev(x + s * way), dev_tok, logp, entropy=entropy, lse=lse)
        values.append(_np(logp + entropy + lse).sum())
    # the quotient: third derivatives times h^2 / 6 (of order 50 |way|^3 1e-4 / 6 at most), values of
    # order 4 known to a few 2^-22 over 2 h
    assert abs((values[0] - values[1]) / (2 * h) - (_np(d) * way).sum()) < 9 * 50 * 1e-4 / 6 + 9 * 4 * 2.0 ** -21 / (2 * h)


# ---------------------------------------------------------------- AdamW
def _adam_tensors(torch, rng, sizes, bits, gtype, ftype, offset=0):
    t = {k: [] for k in ("w", "g", "m", "v", "ms", "vs", "f", "guard")}

    def put(a, dtype):
        flat = torch.full((offset + a.size + 8,), 3.0 if dtype != torch.uint8 else 3, device="cuda", dtype=dtype)
        view = flat[offset:offset + a.size]
        view.copy_(torch.from_numpy(a))
        t["guard"].append((flat, offset, a.size))
        return view
    for n in sizes:
        t["w"].append(put(rng.normal(size=n).astype(np.float32), torch.float32))
        t["g"].append(put((rng.normal(size=n) * np.exp(-6 * rng.random(n))).astype(np.float32), getattr(torch, gtype)))
        t["f"].append(put(np.zeros(n, np.float32), getattr(torch, ftype)) if ftype else None)
        b = -(-n // 256)
        if bits == 8:
            m = rng.integers(0, 256, n).astype(np.uint8)
            m[(m & 127) == 127] = 5
            t["m"].append(put(m, torch.uint8))
            t["v"].append(put(rng.integers(0, 256, n).astype(np.uint8), torch.uint8))
            t["ms"].append(put((rng.random(b) * 1e-3).astype(np.float32), torch.float32))
            t["vs"].append(put((rng.random(b) * 0.3).astype(np.float32), torch.float32))
        else:
            t["m"].append(put((rng.normal(size=n) * 0.1).astype(np.float32), torch.float32))
            t["v"].append(put((rng.random(n) * 0.01).astype(np.float32), torch.float32))
            t["ms"].append(None)
            t["vs"].append(None)
    return t


def _plan(p, t, bits, ftype, decay, horizon):
    return p.AdamW(t["w"], t["m"], t["v"], m_scale=t["ms"] if bits == 8 else None, v_scale=t["vs"] if bits == 8 else None,
                   w_forward=t["f"] if ftype else None, weight_decay=decay, horizon=horizon)


def _guards_hold(t):
    for flat, offset, n in t["guard"]:
        assert (flat[:offset] == 3).all() and (flat[offset + n:] == 3).all()


LR, B1, B2, EPS = 2e-3, 0.9, 0.999, 1e-8


def _f32(t):
    return t.float().cpu().numpy()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gtype,ftype", [("float32", None), ("bfloat16", "bfloat16"), ("float16", "float16"), ("float32", "bfloat16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("sizes,offset", [([1], 0), ([256, 255, 257], 0), ([7, 1000, 0, 33, 4096], 1), ([2048 * 3 + 5, 8, 511], 4), ([100000], 0)])
def test_adamw_step(sizes, offset, gtype, ftype, bits):
    torch, p = _torch()
    rng = np.random.default_rng(sum(sizes) + bits)
    t = _adam_tensors(torch, rng, sizes, bits, gtype, ftype, offset)
    decay, horizon = [0.1 * (k % 2) for k in range(len(sizes))], [float(k) for k in range(len(sizes))]
    plan = _plan(p, t, bits, ftype, decay, horizon)
    gs = torch.tensor(0.37, device="cuda")
    for step in (1, 2, 1000):
        w0, m0, v0 = ([x.cpu().numpy().copy() for x in t[k]] for k in ("w", "m", "v"))
        s0 = [(_f32(a), _f32(b)) if a is not None else None for a, b in zip(t["ms"], t["vs"])]
        plan.step(t["g"], lr=LR, step=step, beta1=B1, beta2=B2, eps=EPS, seed=11, grad_scale=gs)
        for k, n in enumerate(sizes):
            if n == 0:
                continue
            g = _f32(t["g"][k]) * np.float32(0.37)                # one rounding, on both sides
            if bits == 8:
                m32, v32 = O.adamw_read8(m0[k], s0[k][0], v0[k], s0[k][1])
                new = O.adamw_state8(m0[k], s0[k][0], v0[k], s0[k][1], g, B1, B2, 11 + step, k)
                for a, b in zip(new, (t["m"][k], t["ms"][k], t["v"][k], t["vs"][k])):
                    np.testing.assert_array_equal(b.cpu().numpy(), a)
                got = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
                p.adamw_moments(t["m"][k].clone(), t["ms"][k].clone(), t["v"][k].clone(), t["vs"][k].clone(), *got)
                for a, b in zip(O.adamw_read8(*new), got):
                    np.testing.assert_array_equal(b.cpu().numpy(), a)
            else:
                m32, v32 = m0[k], v0[k]
                f = np.float32                                    # every operation rounded, as documented
                np.testing.assert_array_equal(_f32(t["m"][k]), f(B1) * m32 + f(1 - B1) * g)
                np.testing.assert_array_equal(_f32(t["v"][k]), f(B2) * v32 + (f(1 - B2) * g) * g)
            # The moments as the kernel has them (float32, checked bit by bit above), then the update in float64:
            m32, v32 = np.float32(B1) * m32 + np.float32(1 - B1) * g, np.float32(B2) * v32 + (np.float32(1 - B2) * g) * g
            u = (m32.astype(np.float64) / (1 - B1 ** step)) / (np.sqrt(v32.astype(np.float64)) / np.sqrt(1 - B2 ** step) + EPS)
            ref = w0[k].astype(np.float64) * (1 - LR * np.float64(np.float32(decay[k]))) - LR * u
            # u: root, two corrections, their products, sum and division, lr: 16 roundings; w: three
            err_u = 16 * U * np.abs(u)
            tol = LR * err_u + 4 * U * (np.abs(w0[k]) + np.abs(LR * u))
            _close(_np(t["w"][k]), ref, tol)
            if ftype:
                ahead = ref - LR * horizon[k] * u
                rel, ab = _half(ftype)
                _close(_np(t["f"][k]), ahead, tol + LR * horizon[k] * (err_u + 4 * U * np.abs(u)) + (rel + U) * np.abs(ahead) + ab)
    _guards_hold(t)


def test_adamw_many_tensors_equals_one_by_one():
    # more tensors than one launch takes; the 8-bit rounding's stream goes with the place in the list, so compare with 32 bits
    torch, p = _torch()
    rng = np.random.default_rng(0)
    sizes = list(rng.integers(1, 700, 1100))
    a = _adam_tensors(torch, np.random.default_rng(1), sizes, 32, "float32", None)
    b = _adam_tensors(torch, np.random.default_rng(1), sizes, 32, "float32", None)
    _plan(p, a, 32, None, 0.01, 0.0).step(a["g"], lr=LR, step=3)
    for k in range(0, len(sizes), 13):
        p.AdamW([b["w"][k]], [b["m"][k]], [b["v"][k]], weight_decay=0.01).step([b["g"][k]], lr=LR, step=3)
        for q in ("w", "m", "v"):
            assert torch.equal(a[q][k], b[q][k])
    _guards_hold(a)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_device_scalars_and_skipped_steps(bits):
    torch, p = _torch()
    sizes = [300, 5000]
    a = _adam_tensors(torch, np.random.default_rng(2), sizes, bits, "bfloat16", "bfloat16")
    b = _adam_tensors(torch, np.random.default_rng(2), sizes, bits, "bfloat16", "bfloat16")
    pa, pb_ = _plan(p, a, bits, "bfloat16", 0.1, 2.0), _plan(p, b, bits, "bfloat16", 0.1, 2.0)
    lr32 = float(np.float32(LR))
    pa.step(a["g"], lr=lr32, step=7, seed=5)
    pb_.step(b["g"], lr=99.0, step=0, seed=5, dev_lr=torch.tensor(LR, device="cuda"), dev_step=torch.tensor(7, device="cuda"),
             grad_scale=torch.ones((), device="cuda"))
    keys = ("w", "m", "v", "f") + (("ms", "vs") if bits == 8 else ())
    for q in keys:
        for x, y in zip(a[q], b[q]):
            assert torch.equal(x, y), q
    before = {q: [x.clone() for x in a[q]] for q in keys}
    for bad in (float("nan"), float("inf")):
        pa.step(a["g"], lr=LR, step=8, grad_scale=torch.tensor(bad, device="cuda"))
    for q in keys:
        for x, y in zip(a[q], before[q]):
            assert torch.equal(x, y), q


def test_adamw_gradients_that_are_not_finite():
    torch, p = _torch()
    for bits in (32, 8):
        t = _adam_tensors(torch, np.random.default_rng(4), [1000], bits, "float32", None)
        t["g"][0][300] = float("nan")
        t["g"][0][900] = float("inf")
        _plan(p, t, bits, None, 0.0, 0.0).step(t["g"], lr=LR, step=1)
        w = _np(t["w"][0])
        assert np.isnan(w[[300, 900]]).all() and np.isfinite(np.delete(w, [300, 900])).all()
        if bits == 8:
            m, v = torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda")
            p.adamw_moments(t["m"][0], t["ms"][0], t["v"][0], t["vs"][0], m, v)
            nan = np.zeros(1000, bool)
            nan[256:512] = nan[768:] = True                       # the blocks that hold them
            np.testing.assert_array_equal(np.isnan(m.cpu().numpy()), nan)
            np.testing.assert_array_equal(np.isnan(v.cpu().numpy()), nan)
        else:
            assert np.isfinite(np.delete(_np(t["m"][0]), [300, 900])).all()


def test_adamw_fresh_eight_bit_state_and_zero_gradients():
    torch, p = _torch()
    n = 700
    z = lambda dtype, n: torch.zeros(n, dtype=dtype, device="cuda")         # noqa: E731
    w, m, v, ms, vs = torch.ones(n, device="cuda"), z(torch.uint8, n), z(torch.uint8, n), z(torch.float32, 3), z(torch.float32, 3)
    plan = p.AdamW([w], [m], [v], m_scale=[ms], v_scale=[vs])
    plan.step([z(torch.float32, n)], lr=0.1, step=1)
    assert (w == 1).all() and not m.any() and not v.any() and not ms.any() and not vs.any()
    g = torch.zeros(n, device="cuda")
    g[5], g[6] = 1.0, 1e-30                                       # a square below the smallest float32
    plan.step([g], lr=0.1, step=1)
    assert v[5] == 255 and v[6] == 0 and m[5] == 0x7E and abs(float(w[5]) - 0.9) < 1e-6


def test_adamw_refuses_what_does_not_fit():
    torch, p = _torch()
    t = lambda n=100, d=torch.float32: torch.zeros(n, device="cuda", dtype=d)     # noqa: E731
    u8 = lambda n=100: t(n, torch.uint8)                                   # noqa: E731
    big = t(400)
    good = p.AdamW([t()], [t()], [t()])
    for call in (lambda: p.AdamW([t()], [t()], []), lambda: p.AdamW([t()], [t(99)], [t()]), lambda: p.AdamW([t()], [u8()], [u8()]),
                 lambda: p.AdamW([t()], [t()], [t()], m_scale=[t(1)], v_scale=[t(1)]), lambda: p.AdamW([t(d=torch.bfloat16)], [t()], [t()]),
                 lambda: p.AdamW([big[:100]], [big[50:150]], [t()]), lambda: p.AdamW([big[:100], big[:100]], [t(), t()], [t(), t()]),
                 lambda: p.AdamW([big[::4]], [t()], [t()]), lambda: p.AdamW([t(), t()], [t(), t()], [t(), t()], w_forward=[t(), None]),
                 lambda: p.AdamW([t()], [u8()], [u8()], m_scale=[t(2)], v_scale=[t(1)]), lambda: p.AdamW([t()], [t()], [t()], weight_decay=[0.1, 0.2]),
                 lambda: good.step([], lr=0.1, step=1), lambda: good.step([t(99)], lr=0.1, step=1), lambda: good.step([t(d=torch.float64)], lr=0.1, step=1),
                 lambda: good.step([big[::4]], lr=0.1, step=1), lambda: good.step([t()], lr=0.1, step=0), lambda: good.step([t()], lr=-0.1, step=1),
                 lambda: good.step([t().cpu()], lr=0.1, step=1)):
        with pytest.raises(p.PBError) as e:
            call()
        assert e.value.code == -1
    p.AdamW([], [], []).step([], lr=0.1, step=1)


# ---------------------------------------------------------------- calls as programs make them
def test_shapes_that_do_not_fit_are_refused():
    torch, p = _torch()
    f = lambda *n: torch.zeros(*n, device="cuda")                 # noqa: E731
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    scratch = torch.empty(p.embed_scratch_bytes(4, 10, 8), dtype=torch.uint8, device="cuda")
    for call in (lambda: p.embed_forward(f(10, 8), ids, f(4, 7)), lambda: p.embed_forward(f(10, 8), ids, f(5, 8)),
                 lambda: p.embed_forward(f(10, 8).t(), ids, f(4, 10)), lambda: p.embed_forward(f(10, 8), ids.float(), f(4, 8)),
                 lambda: p.embed_forward(f(10, 8), ids, f(4, 8).half()), lambda: p.embed_forward(f(10, 8).double(), ids, f(4, 8).double()),
                 lambda: p.embed_forward(f(10, 8), ids, f(4, 8).cpu()), lambda: p.embed_forward(f(10, 8), ids.cpu(), f(4, 8)),
                 lambda: p.embed_forward(f(10, 8), ids, f(10, 8)[3:7].expand(4, 8)[:, :0]),
                 lambda: p.embed_backward(f(1, 8).expand(4, 8), ids, f(10, 8), scratch),          # a broadcast gradient
                 lambda: p.embed_backward(f(4, 8), ids, f(10, 8), scratch[:64]), lambda: p.embed_backward(f(4, 8), ids, f(10, 8), f(4096)),
                 lambda: p.embed_backward(f(4, 8), ids, f(10, 8).half(), scratch),
                 lambda: p.logprob_forward(f(1, 8).expand(4, 8), ids, f(4)), lambda: p.logprob_forward(f(4, 8), ids, None),
                 lambda: p.logprob_forward(f(4, 8), ids[:3], f(4)), lambda: p.logprob_forward(f(4, 8), ids, f(4).half()),
                 lambda: p.logprob_forward(f(4, 8), ids, f(4), top_logp=f(4, 2), top_ids=torch.zeros(4, 2, dtype=torch.int64, device="cuda")),
                 lambda: p.logprob_forward(f(4, 8), ids, f(4), top_logp=f(4, 9), top_ids=torch.zeros(4, 9, dtype=torch.int32, device="cuda")),
                 lambda: p.logprob_backward(f(4, 8), ids, f(4), f(4, 9), g_logp=f(4)), lambda: p.logprob_backward(f(4, 8), ids, f(4), f(4, 8).half())):
        with pytest.raises(p.PBError) as e:
            call()
        assert e.value.code == -1
    one = f(40)
    with pytest.raises(p.PBError):                                # the same buffer one element further
        p.logprob_backward(one[:32].view(4, 8), ids, f(4), one[1:33].view(4, 8), g_logp=f(4))


def _run_of_all(torch, p, s, stream=0):
    """One training step of a tied one-layer token model; every buffer is the caller's."""
    p.embed_forward(s["fwd"], s["ids"], s["x"], scale=2.0, stream=stream)
    torch.matmul(s["x"], s["fwd"].t(), out=s["logits"])
    p.logprob_forward(s["logits"], s["next"], s["logp"], entropy=s["ent"], lse=s["lse"], stream=stream)
    p.logprob_backward(s["logits"], s["next"], s["lse"], s["logits"], g_logp=s["gl"], g_entropy=s["gh"], entropy=s["ent"], stream=stream)
    torch.matmul(s["logits"].t().float(), s["x"].float(), out=s["dtable"])
    torch.matmul(s["logits"], s["fwd"], out=s["dx"])
    p.embed_backward(s["dx"], s["ids"], s["dtable"], s["scratch"], scale=2.0, accumulate=True, stream=stream)
    s["plan"].step([s["dtable"]], lr=LR, step=0, seed=3, dev_step=s["step"], stream=stream)


def _model(torch, p, bits, seed=0, vocab=1003, dim=72, n=200):
    rng = np.random.default_rng(seed)
    dev = lambda a, d=torch.float32: torch.tensor(a, device="cuda").to(d)    # noqa: E731
    w = dev(rng.normal(size=(vocab, dim)) * 0.1)
    tok = rng.integers(0, vocab, n + 1) // 2
    tok[50] = -1
    s = {"w": w, "fwd": w.bfloat16(), "ids": dev(tok[:-1], torch.int64), "next": dev(tok[1:], torch.int64)}
    e = lambda *n, d=torch.float32: torch.empty(*n, device="cuda", dtype=d)  # noqa: E731
    s.update(x=e(n, dim, d=torch.bfloat16), logits=e(n, vocab, d=torch.bfloat16), logp=e(n), ent=e(n), lse=e(n), dtable=e(vocab, dim),
             dx=e(n, dim, d=torch.bfloat16), scratch=e(p.embed_scratch_bytes(n, vocab, dim), d=torch.uint8), step=dev([1], torch.int64),
             gl=torch.full((n,), -1.0 / n, device="cuda"), gh=torch.full((n,), -0.01 / n, device="cuda"))
    size = vocab * dim
    state = torch.uint8 if bits == 8 else torch.float32
    s["m"], s["v"] = torch.zeros(size, device="cuda", dtype=state), torch.zeros(size, device="cuda", dtype=state)
    s["ms"], s["vs"] = (torch.zeros(-(-size // 256), device="cuda") for _ in range(2))
    kw = dict(m_scale=[s["ms"]], v_scale=[s["vs"]]) if bits == 8 else {}
    s["plan"] = p.AdamW([s["w"]], [s["m"]], [s["v"]], w_forward=[s["fwd"]], weight_decay=0.1, **kw)
    return s, tok


@pytest.mark.parametrize("bits", [32, 8])
def test_a_training_step_of_all_of_them(bits):
    torch, p = _torch()
    s, tok = _model(torch, p, bits)
    w0, f0 = s["w"].double().clone(), s["fwd"].double().clone()
    _run_of_all(torch, p, s)
    # the same step in float64 by autograd, from the bf16 forward weights
    n, f = len(tok) - 1, f0.clone().requires_grad_(True)
    x = torch.where((s["ids"] >= 0)[:, None], 2.0 * f[s["ids"].clamp(min=0)], 0.0)
    lp = torch.log_softmax(x @ f.t(), 1)
    live = s["next"] >= 0
    loss = -(torch.where(live, lp[torch.arange(n), s["next"].clamp(min=0)], 0.0)).sum() / n - 0.01 / n * -(lp.exp() * lp).sum()
    loss.backward()
    # bf16 logits, activations and logit gradients: a few 2^-8 of each of many terms, whose signs are random
    err = (s["dtable"].double() - f.grad).norm() / f.grad.norm()
    assert err < 3 * 2.0 ** -8
    # first step of Adam from zero states: u = g / (|g| + eps'), so w moves by lr in the gradient's direction
    g = s["dtable"].double()
    u = g / (g.abs() + EPS)
    ref = w0 * (1 - LR * float(np.float32(0.1))) - LR * u
    assert ((s["w"].double() - ref).abs() <= LR * 32 * U + 4 * U * w0.abs() + 4 * U * LR).all()
    assert torch.equal(s["fwd"], s["w"].bfloat16())


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_replay_and_do_not_share(bits):
    torch, p = _torch()
    eager, _ = _model(torch, p, bits, seed=1)
    a, _ = _model(torch, p, bits, seed=1)
    b, _ = _model(torch, p, bits, seed=2)
    b_eager, _ = _model(torch, p, bits, seed=2)
    streams, graphs = (torch.cuda.Stream(), torch.cuda.Stream()), []
    for k, s in enumerate((a, b)):                                # torch's products keep a workspace per stream: one stream each
        warm, _ = _model(torch, p, bits, seed=3)
        torch.cuda.synchronize()
        with torch.cuda.stream(streams[k]):
            _run_of_all(torch, p, warm, streams[k].cuda_stream)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=streams[k]):
            _run_of_all(torch, p, s, streams[k].cuda_stream)
            s["step"].add_(1)
        graphs.append(graph)
    for _ in range(3):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()                                    # beside each other
        torch.cuda.synchronize()
        for s in (eager, b_eager):
            _run_of_all(torch, p, s)
            s["step"].add_(1)
    torch.cuda.synchronize()
    for x, y in ((a, eager), (b, b_eager)):
        for k in ("w", "m", "v", "ms", "vs", "logp", "dtable"):
            assert torch.equal(x[k], y[k]), k


def test_calls_on_another_stream_wait_for_it():
    torch, p = _torch()
    stream = torch.cuda.Stream()
    x, ids = torch.randn(5000, 640, device="cuda"), torch.arange(3000, device="cuda") % 5000
    out = torch.empty(3000, 640, device="cuda")
    table = torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
        table.copy_(x)
        p.embed_forward(table, ids, out, stream=stream.cuda_stream)
    stream.synchronize()
    assert torch.equal(out, x[:3000])


def test_long_tables_pass_32_bit_offsets():
    torch, p = _torch()
    vocab, dim = 70_000, 32_768                                   # 2.3e9 elements, 4.6 GB
    table = torch.empty(vocab, dim, device="cuda", dtype=torch.bfloat16)
    table[-1] = 3.0
    table[0] = 2.0
    ids = torch.tensor([vocab - 1, 0], device="cuda")
    out = torch.empty(2, dim, device="cuda", dtype=torch.bfloat16)
    p.embed_forward(table, ids, out)
    assert (out[0] == 3).all() and (out[1] == 2).all()
    scratch = torch.empty(p.embed_scratch_bytes(2, vocab, dim), dtype=torch.uint8, device="cuda")
    p.embed_backward(out, ids, table, scratch, accumulate=True)
    assert (table[-1] == 6).all() and (table[0] == 4).all()
    # the same memory as logits: the last of many long rows
    rows, v = 32_768, 70_000
    x = table.view(rows, v)
    x.zero_()
    x[-1, 69_999] = 20.0
    tok = torch.full((rows,), 69_999, dtype=torch.int32, device="cuda")
    logp, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    p.logprob_forward(x, tok, logp, lse=lse)
    assert abs(float(logp[0]) + np.log(v)) < 1e-4 and abs(float(logp[-1]) + np.log1p((v - 1) * np.exp(-20.0))) < 1e-6
    p.logprob_backward(x, tok, lse, x, g_logp=torch.ones(rows, device="cuda"))
    assert abs(float(x[0, 0]) * v + 1) < 0.01 and 0.0 < float(x[-1, -1]) < 1e-3 and float(x[0, -1]) == 1.0
