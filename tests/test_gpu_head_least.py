"""Gradients of the head whose coefficients are near float32's smallest numbers."""
import pytest
import torch

pytestmark = pytest.mark.gpu

STORE = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("power", [-112, -118, -124])
def test_coefficients_near_the_smallest_numbers(power, dtype):
    import paper_2003_11666_b200 as p
    g = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    h, w, tok = rand(140, 64).to(dtype), (rand(600, 64) * 0.2).to(dtype), torch.randint(0, 600, (140,), generator=g, device="cuda")
    lse = (h.double() @ w.double().T).logsumexp(1).float()
    gl, out = rand(140), []
    for f in (1.0, 2.0 ** power):
        dw = torch.empty(w.shape, device="cuda")
        p.head_logprob_backward(h, w, torch.empty(p.head_scratch_bytes(h, w, True), device="cuda", dtype=torch.uint8), tok, lse, None, dw, g_logp=gl * f)
        out.append(dw.double())
        dh = torch.empty_like(h)
        p.head_logprob_backward(h, w, torch.empty(p.head_scratch_bytes(h, w, True), device="cuda", dtype=torch.uint8), tok, lse, dh, None, g_logp=gl * f)
        out.append(dh.double())
    # A power of two changes no digit, but that there are no numbers below 2^-149 (float16: 2^-24, half of which a rounding is off by): none of the result, and none
    # of the coefficients, each of which is off by 2^-149 at most (as it is given, and as a product): so much of what multiplies them, p or 1 - p and the row of the other
    # operand.  The split of a call's sums is the same for either.
    prob = (h.double() @ w.double().T - lse.double()[:, None]).exp()
    prob.scatter_(1, tok[:, None], 1.0)
    ref = [out[0] * 2.0 ** power, out[1] * 2.0 ** power]
    off = [prob.T @ h.double().abs(), prob @ w.double().abs()]
    for got, want, o in zip(out[2:], ref, off):
        least = 2.0 ** -149 if got is out[2] or dtype is torch.float32 else 2.0 ** -133 if dtype is torch.bfloat16 else 2.0 ** -24
        # a coefficient that lost digits is another coefficient, and sums of other terms round otherwise: by their roundings, see tests/blocks_ref.py
        extra = o * gl.abs().max().item() * 2.0 ** power * (STORE[dtype] * 2 + 2.0 ** -16) * (gl * 2.0 ** power / 2.0 ** power != gl).any().item()
        assert bool(((got - want).abs() <= least + 2.0 ** -149 * o + extra).all())
