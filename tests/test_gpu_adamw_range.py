"""AdamW steps whose second moments or eps are near float32's smallest numbers, on the GPU against float64."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LR, B1, B2 = 2e-3, 0.9, 0.999


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-30, 1e-20, 1e-15, 1e-10, 1e-8])
def test_update_of_tiny_second_moments(eps, offset):
    # gradients from 1e-21 to 1: squares down to 1e-45, roots of numbers below 2^-126 among them
    import torch
    import paper_2003_11666_b200 as p
    rng = np.random.default_rng(7)
    n = 3001
    g = (10.0 ** rng.uniform(-21, 0, n) * rng.choice([-1.0, 1.0], n)).astype(np.float32)
    m0 = (g * rng.uniform(0.5, 1.5, n)).astype(np.float32)
    v0 = (g.astype(np.float64) ** 2 * rng.uniform(0.5, 1.5, n)).astype(np.float32)
    w0 = rng.normal(size=n).astype(np.float32)

    def put(a):
        flat = torch.zeros(n + 8, device="cuda")
        flat[offset:offset + n].copy_(torch.from_numpy(a))
        return flat[offset:offset + n]
    w, m, v = put(w0), put(m0), put(v0)
    f = np.float32
    for step in (1, 50):
        start = w.cpu().numpy().astype(np.float64)
        m1 = f(B1) * m.cpu().numpy() + f(1 - B1) * g
        v1 = f(B2) * v.cpu().numpy() + (f(1 - B2) * g) * g
        p.AdamW([w], [m], [v]).step([put(g)], lr=LR, step=step, beta1=B1, beta2=B2, eps=eps)
        np.testing.assert_array_equal(m.cpu().numpy(), m1)
        np.testing.assert_array_equal(v.cpu().numpy(), v1)
        eps32 = np.float64(f(eps))
        with np.errstate(divide="ignore", invalid="ignore"):
            u = (m1.astype(np.float64) / (1 - B1 ** step)) / (np.sqrt(v1.astype(np.float64)) / np.sqrt(1 - B2 ** step) + eps32)
        live = v1 > 0                                              # 0 / 0 and x / 0 otherwise, as the formula says, with eps = 0
        live |= eps32 > 1e-36
        # u: as in the step's other tests, 16 roundings; a denominator below 2^-126 has lost digits of its own
        tol = LR * 16 * U * np.abs(u) + 4 * U * (np.abs(start) + np.abs(LR * u))
        got = w.cpu().numpy().astype(np.float64)
        bad = ~(np.abs(got - (start - LR * u)) <= tol) & live
        assert not bad.any(), (int(bad.sum()), g[bad][:4], v1[bad][:4], got[bad][:4], (start - LR * u)[bad][:4])
        w.copy_(torch.from_numpy(w0))


def test_eight_bit_step_of_tiny_gradients_with_no_eps():
    import torch
    import paper_2003_11666_b200 as p
    n = 700
    z = lambda k, d: torch.zeros(k, device="cuda", dtype=d)        # noqa: E731
    w, m, v, ms, vs = torch.ones(n, device="cuda"), z(n, torch.uint8), z(n, torch.uint8), z(3, torch.float32), z(3, torch.float32)
    g = torch.full((n,), 1e-18, device="cuda")                     # v = 1e-39: below 2^-126
    p.AdamW([w], [m], [v], m_scale=[ms], v_scale=[vs]).step([g], lr=0.125, step=1, beta1=B1, beta2=B2, eps=0.0)
    # u = g / |g| up to the digits of v, a number of some 2^20 steps of 2^-149
    assert (w - 0.875).abs().max() < 0.125 * 2.0 ** -18
