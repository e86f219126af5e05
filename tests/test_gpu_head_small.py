"""Heads of float32 numbers far below 1, as a table that has just been laid out may hold."""
import pytest
import torch

pytestmark = pytest.mark.gpu


# dhidden is as small, and finite
@pytest.mark.parametrize("power", [-90, -105, -112])
def test_heads_of_very_small_numbers(power):
    import paper_2003_11666_b200 as p
    g = torch.Generator(device="cuda").manual_seed(570)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    h, w, gl = rand(70, 48), rand(500, 48) * 2.0 ** power, rand(70)
    tok = torch.randint(0, 500, (70,), generator=g, device="cuda")
    byte = lambda back: torch.empty(p.head_scratch_bytes(h, w, back), device="cuda", dtype=torch.uint8)      # noqa: E731
    lse, dh, dw = torch.empty(70, device="cuda"), torch.full_like(h, 3.0), torch.full_like(w, 3.0)
    p.head_logprob_forward(h, w, byte(False), lse=lse)
    p.head_logprob_backward(h, w, byte(True), tok, lse, dh, dw, g_logp=gl)
    assert bool(torch.isfinite(dh).all()) and bool((dh != 0).any(1).all())
    big = w * 2.0 ** -power                                       # p is 1 / 500 of either
    prob = torch.full((70, 500), 1 / 500, device="cuda", dtype=torch.float64)
    d = -gl.double()[:, None] * prob
    d.scatter_add_(1, tok[:, None], gl.double()[:, None])
    ref = d @ big.double()
    # d to 2^-19 of itself (logarithms of 500 in float32 and their exponentials), sums as in blocks_ref, elements of the head by their planes: 2^-39 of a group's
    # largest, which is 2^-120 at least
    tol = (d.abs() @ big.double().abs()) * 2.0 ** -16 + 500 * 2.0 ** -37 * (big.abs().max() + 2.0 ** max(-120 + 15 - power, -60)) * 2 * gl.abs().double()[:, None]
    assert bool(((dh.double() * 2.0 ** -power - ref).abs() <= tol).all())
