"""The plain float64 forms against torch's autograd, and dropout's generator against its definition in whole numbers."""
import numpy as np
import torch

from tests import blocks_ref as R


def test_head_matches_autograd():
    g = torch.Generator().manual_seed(1)
    h = torch.randn(7, 5, generator=g, dtype=torch.float64, requires_grad=True)
    w = torch.randn(11, 5, generator=g, dtype=torch.float64, requires_grad=True)
    tok = torch.tensor([0, 10, 3, -1, 2, 2, 11])
    gl, ge, gz = (torch.randn(7, generator=g, dtype=torch.float64) for _ in range(3))
    lp = torch.log_softmax(h @ w.T * 0.7, 1)
    ok = (tok >= 0) & (tok < 11)
    at = torch.where(ok, lp[torch.arange(7), tok.clamp(0, 10)], 0.0)
    lse, ent = torch.logsumexp(h @ w.T * 0.7, 1), -(lp.exp() * lp).sum(1)
    (at * gl + ent * ge + lse * gz).sum().backward()
    logp, entropy, z, _ = R.head_forward(h.detach(), w.detach(), tok, 0.7)
    for a, b in ((logp, at), (entropy, ent), (z, lse)):
        np.testing.assert_allclose(a.numpy(), b.detach().numpy(), rtol=1e-12, atol=1e-13)
    _, dh, dw, _ = R.head_backward(h.detach(), w.detach(), tok, 0.7, z, entropy, gl, ge, gz)
    np.testing.assert_allclose(dh.numpy(), h.grad.numpy(), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(dw.numpy(), w.grad.numpy(), rtol=1e-10, atol=1e-12)


def test_join_matches_autograd():
    g = torch.Generator().manual_seed(2)
    rand = lambda *n: torch.randn(*n, generator=g, dtype=torch.float64)        # noqa: E731
    for post, per, p in ((True, 3, 0.25), (False, 7, 0.0), (True, 1, 0.5)):
        x, u, gate, a, b = rand(7, 6), rand(7, 6), rand(-(-7 // per), 6), rand(6), rand(6)
        factor = R.keep(5, 2, p, 7, 6) if p else None
        leaves = [t.requires_grad_(True) for t in (x, u, gate, a, b)]
        y, h, rp, rr = R.join_forward(x, u, gate, per, a if post else None, b, 0.8, 1e-3, factor)
        dy, dh = rand(7, 6), rand(7, 6)
        ((y * dy).sum() + (h * dh).sum()).backward()
        dx, du, dg, da, db = (t.grad for t in leaves)
        det = [t.detach() for t in leaves]
        out = R.join_backward(y.detach(), det[1], dy, dh, det[2], per, det[3] if post else None, det[4], rp.detach() if post else None, rr.detach(), 0.8, factor)
        for k, ref in (("dx", dx), ("du", du), ("dgate", dg), ("dpost", da), ("dpre", db)):
            if k in out:
                np.testing.assert_allclose(out[k].numpy(), ref.numpy(), rtol=1e-9, atol=1e-11)


def test_generator_in_whole_numbers():
    def splitmix(base, counter):
        m = (1 << 64) - 1
        z = (base + (counter + 1) * 0x9E3779B97F4A7C15) & m
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & m
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & m
        return z ^ (z >> 31)
    assert splitmix(0, 0) == 0xE220A8397B1DCDAF               # first output of the published generator from state 0
    for seed, offset, p in ((0, 0, 0.5), (2 ** 64 - 1, 7, 0.1), (123456789012345, 2 ** 62, 0.999)):
        f = R.keep(seed, offset, p, 5, 7).reshape(-1)
        drop = round(p * 65536)
        base = splitmix(seed, offset)
        for i in range(35):
            kept = (splitmix(base, i // 4) >> (16 * (i % 4))) & 0xFFFF
            assert f[i] == (65536 / (65536 - drop) if kept >= drop else 0.0)


def test_generator_keeps_the_share_and_mixes_its_streams():
    a, b, c = R.keep(3, 1, 0.3, 512, 512) > 0, R.keep(3, 2, 0.3, 512, 512) > 0, R.keep(4, 1, 0.3, 512, 512) > 0
    n = 512 * 512
    five = 5 * (0.3 * 0.7 / n) ** 0.5                          # five standard deviations of a share of n draws
    for x in (a, b, c):
        assert abs(float(x.double().mean()) - 0.7) < five + 2.0 ** -17
    for x, y in ((a, b), (a, c), (a[:, 1:], a[:, :-1]), (a[1:], a[:-1])):
        both = float((x & y).double().mean())
        assert abs(both - 0.49) < 5 * (0.49 * 0.51 / (n - 512)) ** 0.5 + 2.0 ** -16
