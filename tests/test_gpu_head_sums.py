"""How far the sums of a logit's products may drift: tighter than tests/blocks_ref.py, for what the kernels do."""
import pytest
import torch

from tests import blocks_ref as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _values(h, w, tok, it=1.0):
    import paper_2003_11666_b200 as p
    out = [torch.empty(h.shape[0], device="cuda") for _ in range(3)]
    sc = torch.empty(p.head_scratch_bytes(h, w), device="cuda", dtype=torch.uint8)
    p.head_logprob_forward(h, w, sc, tok, out[0], entropy=out[1], lse=out[2], inv_temperature=it)
    return out


def _logit_error(hidden, weight, it):
    """As R.head_logit_error of 16-bit operands, whose sums of more than 1024 columns leave the tensor core every 1024 (64 steps) and are added up in float32: U of the
    sum for each part."""
    s = hidden.double().abs() @ weight.double().abs().T * it
    n = hidden.shape[1]
    return s * ((min(n, 1024) / 32 + 4) * 2.0 ** -22 + (-(-n // 1024) + 5) * U)


# terms of one sign drift the most: what is cut off always has the same sign
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("rows", [5, 150])
@pytest.mark.parametrize("dim", [512, 1024, 1032, 4100, 9000])
def test_long_rows_of_16_bits(dim, rows, dtype, monkeypatch):
    monkeypatch.setattr(R, "head_logit_error", _logit_error)
    g = torch.Generator(device="cuda").manual_seed(dim + rows)
    rand = lambda *n: torch.rand(*n, generator=g, device="cuda")   # noqa: E731
    tok = torch.randint(0, 300, (rows,), generator=g, device="cuda")
    for low in (0.5, -0.5):                                         # of one sign, and of both
        h, w = ((rand(n, dim) + low).to(dtype) for n in (rows, 300))
        got = _values(h, w, tok)
        rl, re, rz, _ = R.head_forward(h, w, tok, 1.0)
        for a, b, tol in zip(got, (rl, re, rz), R.head_forward_error(h, w, tok, 1.0)):
            assert bool(((a.double() - b).abs() <= tol).all()), float(((a.double() - b).abs() / tol).max())


@pytest.mark.parametrize("dtype,rows", [(torch.float32, 1), (torch.float32, 4), (torch.bfloat16, 1), (torch.bfloat16, 2), (torch.float16, 2)], ids=str)
@pytest.mark.parametrize("dim", [1024, 2048])
def test_sums_of_a_few_rows_round_to_nearest(dim, rows, dtype):
    # terms of one sign, where sums that are cut off drift the most: by the order of 2^-24 per step, all in one direction; a temperature that leaves every token its share
    g = torch.Generator(device="cuda").manual_seed(dim + rows)
    h, w = ((torch.rand(n, dim, generator=g, device="cuda") + 0.5).to(dtype) for n in (rows, 4096))
    z = h.double() @ w.double().T * 0.1
    tok = torch.randint(0, 4096, (rows,), generator=g, device="cuda")
    _, _, lse = _values(h, w, tok, 0.1)
    ref = z.logsumexp(1)
    p = (z - ref[:, None]).exp()
    # A logit of n terms is added up in 64 chains of n / 64, which meet in six more additions: each rounding is off by at most U of the sum that it leaves,
    # to either side, so that its variance is a third of that squared at most; lse takes the mean of the logits' errors under p.  Six deviations of that, the rounding of
    # lse, and of its sum: exponentials to 2^-22 of exponents below 32 that are rounded to U and off by U by their float32 factor, ten additions of U
    spread = (((dim / 64 + 7) / 3) ** 0.5 * U * z.amax(1)) * p.square().sum(1).sqrt()
    tol = 6 * spread + U * ref + 2.0 ** -22 + 2 * U * 32 + 10 * U
    err = (lse.double() - ref).abs()
    assert bool((err <= tol).all()), (err / tol).tolist()


# float32 operands that run on the tensor cores: single blocks and pairs
@pytest.mark.parametrize("rows", [5, 150])
@pytest.mark.parametrize("dim", [256, 1024, 2048])
def test_float32_sums_drift_by_no_more_than_a_few_steps(dim, rows):
    # terms of one sign again.  What a step of the tensor core's sum drops is half of the sum's last place on average, and a sum leaves it after 24 steps at most:
    # it grows by a 24th of itself with each
    part = torch.arange(1, 25, dtype=torch.float64) / 24
    g = torch.Generator(device="cuda").manual_seed(dim + rows)
    h, w = ((torch.rand(n, dim, generator=g, device="cuda") + 0.5) for n in (rows, 4096))
    scale = 102.4 / dim
    z = h.double() @ w.double().T * scale
    tok = torch.randint(0, 4096, (rows,), generator=g, device="cuda")
    _, _, lse = _values(h, w, tok, scale)
    ref = z.logsumexp(1)
    per_part = 128.0                                                # a part is the sum of 128 columns of numbers near 1, of any binade's place
    drift = 0.5 * 2.0 ** -23 * float((2.0 ** torch.floor(torch.log2(part * per_part))).sum()) / per_part
    # 1.6 times that for logits that differ from the mean, and lse's own: see above
    tol = 1.6 * drift * z.mean(1) + U * ref + 2.0 ** -22 + 2 * U * 32 + 10 * U
    err = (lse.double() - ref).abs()
    assert bool((err <= tol).all()), ((err / tol).max(), drift)
