"""Logits far from zero: logsumexps are good to their own rounding, and in the gradients the probability of a token is exp(z - lse) of the lse that is given, to
float32's last digits of the difference, not of z and lse."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("it", [1.0, 0.7, 1.3])
@pytest.mark.parametrize("rows", [3, 200])
@pytest.mark.parametrize("level", [0.0, 15.0, 130.0, -1000.0, 4000.0])
def test_probabilities_far_from_zero(level, rows, it):
    import paper_2003_11666_b200 as p
    vocab, dim = 96, 8
    g = torch.Generator(device="cuda").manual_seed(rows)
    # one column counts, and every logit is a number of float32 (its two planes hold it): level + k / 64
    h, w = torch.zeros(rows, dim, device="cuda"), torch.zeros(vocab, dim, device="cuda")
    h[:, 0] = 1.0
    w[:, 0] = level + torch.randint(-200, 200, (vocab,), generator=g, device="cuda") / 64
    z = h.double() @ w.double().T * it
    lse = (z.logsumexp(1) + 0.01 * torch.rand(rows, generator=g, device="cuda")).float()
    entropy, ge, gz = torch.full((rows,), 2.0, device="cuda"), torch.full((rows,), 0.5, device="cuda"), torch.full((rows,), 1.5, device="cuda")
    tok = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    gl = torch.rand(rows, generator=g, device="cuda")
    lp = z - lse.double()[:, None]
    for parts in ((None, None, gz), (gl, None, None), (gl, ge, gz)):
        dh, dw = torch.empty_like(h), torch.empty_like(w)
        sc = torch.empty(p.head_scratch_bytes(h, w, True), device="cuda", dtype=torch.uint8)
        p.head_logprob_backward(h, w, sc, tok, lse, dh, dw, g_logp=parts[0], g_entropy=parts[1], entropy=entropy, g_lse=parts[2], inv_temperature=it)
        c = [torch.zeros(rows, 1, device="cuda", dtype=torch.float64) if x is None else x.double()[:, None] for x in parts]
        prob = lp.exp()
        d = prob * (c[2] - c[0]) - c[1] * prob * (lp + entropy.double()[:, None])
        d.scatter_add_(1, tok[:, None], c[0])
        d *= it
        # the exponent in units of log 2 is rounded once (U of itself), the factor for them is a float32 (U of the exponent, since lse is taken by the same one), the
        # exponential is good to 2^-22; what multiplies p takes four roundings (three products, the correction of lse) and is known to U of its terms; d is summed
        # over rows / 128 + 5 parts of at most 48 steps of 2^-22, and stored.  Where 1 - p is formed, p itself counts
        size = it * (c[2].abs() + c[0].abs() + c[1] * (lp.abs() + 2.0))
        off = prob * size * (2.0 ** -22 + 2 * U * lp.abs() + 8 * U) + prob * it * c[1] * 2 * U * lp.abs() + d.abs() * 4 * U
        tol = off.sum(0) + d.abs().sum(0) * (28 * 2.0 ** -22 * (rows > 4) + (rows / 128 + 7) * U)
        err = (dw[:, 0].double() - d.sum(0)).abs()
        assert bool((err <= tol).all()), float((err / tol).max())


# a few rows, a tile, pairs of tiles; the reference of a row's sum is a float32 that stands for the logit it was formed of
@pytest.mark.parametrize("it", [1.0, 0.79, 1.57])
@pytest.mark.parametrize("rows", [3, 20, 200])
@pytest.mark.parametrize("level", [0.0, 15.0, -1000.0, 4000.0, 30000.0])
def test_logsumexps_far_from_zero(level, rows, it):
    import paper_2003_11666_b200 as p
    vocab, dim = 96, 8
    g = torch.Generator(device="cuda").manual_seed(rows)
    h, w = torch.zeros(rows, dim, device="cuda"), torch.zeros(vocab, dim, device="cuda")
    h[:, 0] = 1.0
    w[:, 0] = level + torch.randint(-200, 200, (vocab,), generator=g, device="cuda") / 64
    tok = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    logp, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    p.head_logprob_forward(h, w, torch.empty(p.head_scratch_bytes(h, w), device="cuda", dtype=torch.uint8), tok, logp, lse=lse, inv_temperature=it)
    z = h.double() @ w.double().T * it
    ref = z.logsumexp(1)
    # the result's rounding (the logarithm is taken in 64 bits; its sum: exponentials to 2^-22 of exponents below 16 that are rounded to U and off by U by their float32 factor)
    tol = U * ref.abs() + 2.0 ** -21 + 2 * U * 16
    assert bool(((lse.double() - ref).abs() <= tol).all()), float(((lse.double() - ref).abs() / tol).max())
    want = z.gather(1, tok[:, None])[:, 0] - ref
    assert bool(((logp.double() - want).abs() <= 2.0 ** -21 + 4 * U * 16 + U * want.abs()).all())
