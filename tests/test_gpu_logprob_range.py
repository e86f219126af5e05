"""Log probabilities over the whole range of sizes, masks and temperatures that are accepted, on the GPU against the
float64 oracle, with the tolerances that tests/test_gpu_tokens.py derives."""
import numpy as np
import pytest

from oracle import tokens as O
from tests.test_gpu_tokens import U, _close, _logprob_case, _logprob_gradient, _logprob_tolerance, _matrix, _np, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [262145 + 512, 300000, 524287, 600001, 700003])
@pytest.mark.parametrize("kind", ["normal", "ties"])
def test_alternatives_of_float32_rows_with_many_segments(vocab, kind):
    # more maxima than the selection keeps in registers, by rows of one block and of a cluster
    for rows in (1, 3, 300):
        if rows * vocab > 4e7 and kind == "ties":
            continue
        for k in (1, 20) if rows < 300 else (20,):
            torch, p = _torch()
            if rows < 300:
                _logprob_case(rows, vocab, "float32", kind, 1.0, k, offset=rows)
                continue
            x = torch.randn(rows, vocab, device="cuda")
            top, ids = torch.empty(rows, k, device="cuda"), torch.empty(rows, k, dtype=torch.int32, device="cuda")
            p.logprob_forward(x, top_logp=top, top_ids=ids)
            assert torch.equal(ids.long(), torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k])


def test_alternatives_of_a_long_float32_row_that_is_not_finite():
    torch, p = _torch()
    vocab, k = 300000, 20
    x = torch.randn(4, vocab, device="cuda")
    x[0, 7] = float("nan")
    x[1] = -float("inf")
    x[2] = torch.finfo(torch.float32).min
    x[3] = float("nan")
    lse, top, ids = torch.empty(4, device="cuda"), torch.empty(4, k, device="cuda"), torch.empty(4, k, dtype=torch.int32, device="cuda")
    p.logprob_forward(x, lse=lse, top_logp=top, top_ids=ids)
    assert (ids[[0, 1, 3]] == -1).all() and torch.equal(ids[2].cpu(), torch.arange(k, dtype=torch.int32))
    assert top[[0, 3]].isnan().all() and (top[1] == -float("inf")).all() and lse[[0, 3]].isnan().all()
    # equal logits: each has the logarithm of 1 / vocab, rounded once
    assert np.abs(top[2].double().cpu().numpy() + np.log(vocab)).max() <= np.log(vocab) * 2.0 ** -22


def _masked_rows(rng, vocab, mask, dtype):
    """Rows whose finite mask lies where a warp or a row meets it first, last, or alone."""
    x = rng.normal(size=(9, vocab)) * 2.5
    at = np.arange(vocab)
    x[0, :vocab * 3 // 5] = mask                                  # whole leading pieces
    x[1, vocab * 2 // 5:] = mask                                  # whole trailing pieces
    x[2] = mask
    x[2, vocab // 2] = 0.25                                       # one token left
    x[3] = mask                                                   # none left
    x[4, :5] = mask                                               # the logits before a row's first aligned one
    x[5, (at >> 10) % 2 == 1] = mask                              # every other piece
    x[6, rng.random(vocab) < 0.5] = mask
    x[7, at % 2 == 0] = mask                                      # two masks, and nothing else
    x[7, at % 2 == 1] = mask * 1.5 if abs(mask) < 1e37 and dtype != "float16" else mask
    x[8] += -mask if abs(mask) < 1e36 and dtype != "float16" else 0.0     # far above zero
    return x


def _check_values(x, dtype, it, k, offset=0):
    torch, p = _torch()
    rows, vocab = x.shape
    flat, dev = _matrix(torch, x, dtype, None, offset)
    xs = _np(dev)
    tok = np.arange(rows) * 7919 % vocab
    f = lambda *n: torch.full(n, 9.0, device="cuda")              # noqa: E731
    logp, entropy, lse, top, ids = f(rows), f(rows), f(rows), f(rows, k), torch.full((rows, k), 9, dtype=torch.int32, device="cuda")
    p.logprob_forward(dev, torch.tensor(tok, device="cuda"), logp, entropy=entropy, lse=lse, top_logp=top, top_ids=ids, inv_temperature=it)
    rl, re, rz, rt, ri = O.logprob_forward(xs, tok, it, k)
    tz, te = _logprob_tolerance(xs, it, rows)
    big = float(np.finfo(np.float32).max)                         # what float32 cannot hold is infinite
    for got, ref, tol in ((lse, rz, tz), (logp, rl, tz), (entropy, re, te), (top, rt, tz[:, None])):
        ref = np.where(np.abs(ref) > big * (1 + U), np.copysign(np.inf, ref), ref)
        with np.errstate(invalid="ignore"):
            _close(_np(got), ref, tol + np.where(np.isfinite(ref), 2 * U * np.abs(ref), 0.0))
    np.testing.assert_array_equal(ids.cpu().numpy(), ri)
    return dev, tok, rl, re, rz


MASKS = [-1e5, -1e9, -4.5e9, -1e10, -1e12, -1e15, -1e20, -1e30, -1e32, -7e35, -2e36, -1e38]


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab,offset", [(300, 0), (300, 3), (40000, 0), (40001, 5), (131075, 1)])
def test_values_of_rows_with_finite_masks(vocab, offset, dtype, mask):
    rng = np.random.default_rng(vocab)
    x = _masked_rows(rng, vocab, mask, dtype)
    for it in (1.0, 0.7, 1.3):
        _check_values(x, dtype, it, 4, offset)


@pytest.mark.parametrize("it", [1e-38, 1e-6, 1e-3, 1e3, 1e6, 1e9, 1e12, 1e20, 1e30, 3e38])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("vocab", [300, 40001, 131075])
def test_values_at_temperatures_far_from_one(vocab, dtype, it):
    rng = np.random.default_rng(vocab)
    x = np.concatenate([_masked_rows(rng, vocab, float(np.finfo(np.float16).min), dtype), 20.0 * rng.normal(size=(20, vocab))])
    x[-1] = 0.0
    _check_values(x, dtype, it, 4, 1)


def test_values_of_many_short_rows_with_finite_masks():
    # more rows than blocks are resident: two warps each
    rng = np.random.default_rng(5)
    for dtype in ("float32", "bfloat16"):
        x = np.tile(_masked_rows(rng, 3001, -1e10, dtype), (90, 1))
        _check_values(x, dtype, 0.7, 4)


FULL_MASKS = [-1e6, -1e9, -1e10, -1e12, -1e30, -3e38, 1e10]


@pytest.mark.parametrize("it", [1.0, 0.7, 1.3, 1e-3])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab,offset", [(300, 0), (5001, 3)])
def test_gradient_of_rows_whose_logsumexp_is_large(vocab, offset, dtype, it):
    # A float32 lse of 1e10 is a multiple of 1024, so exp(it x - lse) of such a row could be anything.  It is a
    # probability all the same: rows that get no gradient pass none on, others none beyond their factor.
    torch, p = _torch()
    rows = len(FULL_MASKS)
    _, dev = _matrix(torch, np.repeat(np.array(FULL_MASKS)[:, None], vocab, 1), dtype, None, offset)
    _, d = _matrix(torch, np.zeros((rows, vocab)), dtype, None, offset)
    tok = torch.full((rows,), vocab // 2, device="cuda")
    logp, lse, entropy = (torch.empty(rows, device="cuda") for _ in range(3))
    p.logprob_forward(dev, tok, logp, lse=lse, entropy=entropy, inv_temperature=it)
    # 3e38 times 1.3 is beyond float32: that row's lse is -inf, and it has no gradient
    assert torch.equal(torch.isfinite(lse), (dev[:, 0].double() * it).abs() < 3.4e38) and torch.isfinite(entropy).all()
    full = lambda v: torch.full((rows,), v, device="cuda")        # noqa: E731
    for where in (d, dev.clone()):                                # apart, and over the logits themselves
        same = where is not d
        src = where if same else dev
        p.logprob_backward(src, tok, lse, where, g_logp=full(0.0), g_entropy=full(0.0), entropy=entropy, g_lse=full(0.0), inv_temperature=it)
        assert (where == 0).all()
    p.logprob_backward(dev, None, lse, d, g_lse=full(0.0), inv_temperature=it)
    assert (d == 0).all()
    p.logprob_backward(dev, tok, lse, d, g_logp=full(-2.0), g_lse=full(0.5), inv_temperature=it)
    got = _np(d)
    # 0 <= p <= 1; the store's rounding and those of the products
    assert np.isfinite(got).all() and (np.abs(got) <= 2.5 * it * (1 + 2.0 ** -7)).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shift", [3e4, 4e4, -1e5, 1e5])
@pytest.mark.parametrize("vocab,offset", [(300, 0), (5001, 3)])
def test_gradient_of_rows_far_from_zero(vocab, offset, shift, dtype):
    torch, p = _torch()
    rng = np.random.default_rng(3)
    x = rng.normal(size=(5, vocab)) * 2.5 + shift
    x[1, vocab // 3] += 9.0
    for it in (1.0, 0.7):
        _, dev = _matrix(torch, x, dtype, None, offset)
        tok = rng.integers(0, vocab, 5)
        _logprob_gradient(torch, p, dev, torch.tensor(tok, device="cuda"), tok, it, dtype, False, None, offset)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab,offset", [(300, 0), (40001, 5)])
def test_entropy_gradient_of_masked_logits_is_zero_at_any_scale(vocab, offset, dtype):
    # a masked logit has p = 0: its gradient is 0, however large the factor beside p is
    torch, p = _torch()
    rng = np.random.default_rng(1)
    x = rng.normal(size=(6, vocab))
    mask = np.array([-np.inf, -np.inf, -1e9, -1e30, -3e38, -1e5])
    hit = rng.random((6, vocab)) < 0.4
    hit[:, 1] = False
    x = np.where(hit, mask[:, None], x)
    _, dev = _matrix(torch, x, dtype, None, offset)
    lse, entropy, d = torch.empty(6, device="cuda"), torch.empty(6, device="cuda"), torch.empty_like(dev)
    xs = _np(dev)
    for it, scale in ((1.0, 1.0), (1.0, 1e9), (1.0, 1e30), (1e6, 1e3), (1e9, 1.0)):
        p.logprob_forward(dev, lse=lse, entropy=entropy, inv_temperature=it)
        p.logprob_backward(dev, None, lse, d, g_entropy=torch.full((6,), scale, device="cuda"), entropy=entropy, inv_temperature=it)
        got = _np(d)
        assert np.isfinite(got).all() and (got[hit] == 0).all(), (it, scale)
        if it == 1.0:
            z, h = _np(lse)[:, None], _np(entropy)[:, None]
            lp = xs - z
            ref = -scale * np.exp(lp) * (np.where(hit, 0.0, lp) + h)
            # p: 2^-20 of itself; the bracket: a few roundings of |log p| + H; the stores's rounding
            tol = scale * np.exp(lp) * (np.where(hit, 0.0, np.abs(lp)) + h) * 2.0 ** -19 + (2.0 ** -8 if dtype == "bfloat16" else U) * np.abs(ref)
            _close(got, ref, tol)
