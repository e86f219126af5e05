"""Heads whose rows are not all alike: vocabularies padded with rows of zeros, and heads of zeros.
Bounds are derived in tests/blocks_ref.py."""
import pytest
import torch

from tests import blocks_ref as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _gradients(h, w, tok, gl):
    import paper_2003_11666_b200 as p
    byte = lambda back: torch.empty(p.head_scratch_bytes(h, w, back), device="cuda", dtype=torch.uint8)      # noqa: E731
    n = h.shape[0]
    logp, entropy, lse = (torch.empty(n, device="cuda") for _ in range(3))
    p.head_logprob_forward(h, w, byte(False), tok, logp, entropy=entropy, lse=lse)
    dh, dw = torch.full_like(h, 3.0), torch.full_like(w, 3.0)
    p.head_logprob_backward(h, w, byte(True), tok, lse, dh, dw, g_logp=gl, g_entropy=0.1 * gl, entropy=entropy)
    return logp, entropy, lse, dh, dw


def _check(h, w, tok, gl):
    logp, entropy, lse, dh, dw = _gradients(h, w, tok, gl)
    rl, re, rz, _ = R.head_forward(h, w, tok, 1.0)
    for got, ref, tol in zip((logp, entropy, lse), (rl, re, rz), R.head_forward_error(h, w, tok, 1.0)):
        assert bool(((got.double() - ref).abs() <= tol).all())
    args = (h, w, tok, 1.0, lse, entropy, gl, 0.1 * gl, None)
    _, rh, rw, _ = R.head_backward(*args)
    eh, ew = R.head_backward_error(*args, 0, U)
    for got, ref, tol in ((dh, rh, eh), (dw, rw, ew)):
        off = (got.double() - ref).abs()
        assert bool((off <= tol).all()), (float((off / tol).max()), float(off.max()), float(ref.abs().max()))


def _case(rows, vocab, dim, size, zeros):
    g = torch.Generator(device="cuda").manual_seed(rows + vocab)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    h, w = rand(rows, dim), rand(vocab, dim) * size
    for a, b in zeros:
        w[a:b] = 0.0
    return h, w, torch.randint(0, vocab, (rows,), generator=g, device="cuda"), rand(rows)


# rows of zeros at the end and in the middle, a whole group of 32 of them or more; all but one group; none of a whole group
@pytest.mark.parametrize("size", [0.02, 0.002])
@pytest.mark.parametrize("rows,vocab,dim,zeros", [(60, 1024, 96, [(992, 1024)]), (60, 1000, 96, [(300, 400), (957, 1000)]), (200, 1500, 72, [(1400, 1500)]),
                                                  (9, 700, 61, [(0, 640), (672, 700)]), (300, 600, 33, [(40, 60)])])
def test_rows_of_zeros(rows, vocab, dim, zeros, size):
    _check(*_case(rows, vocab, dim, size, zeros))


def test_rows_of_zeros_in_a_piece_of_their_own():
    # 8200 rows: pieces of 8192 tokens, of which the last is all zeros
    _check(*_case(8200, 16600, 16, 0.02, [(8000, 16600)]))


@pytest.mark.parametrize("rows", [5, 140])
def test_a_head_of_zeros(rows):
    h, w, tok, gl = _case(rows, 300, 40, 1.0, [(0, 300)])
    logp, entropy, lse, dh, dw = _gradients(h, w, tok, gl)
    ref = torch.log(torch.tensor(300.0, dtype=torch.float64)).item()
    for got, want in ((logp, -ref), (entropy, ref), (lse, ref)):
        assert bool(((got.double() - want).abs() < 2.0 ** -18).all())
    assert bool((dh == 0).all())
    _check(h, w, tok, gl)
