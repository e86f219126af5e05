"""The oracle's token operators against torch CPU autograd, torch's AdamW and central differences."""
import numpy as np
import pytest
import torch

from oracle import tokens as O


def test_embedding_and_its_gradient_match_autograd():
    rng = np.random.default_rng(1)
    table, ids, scale = rng.normal(size=(13, 6)), rng.integers(0, 13, 40), 2.5
    w = torch.tensor(table, requires_grad=True)
    out = torch.nn.functional.embedding(torch.tensor(ids), w, padding_idx=4) * scale
    dout = rng.normal(size=(40, 6))
    out.backward(torch.tensor(dout))
    np.testing.assert_allclose(O.embed_forward(table, ids, scale), out.detach().numpy(), rtol=1e-14)
    np.testing.assert_allclose(O.embed_backward(dout, ids, 13, scale, padding=4), w.grad.numpy(), rtol=1e-12, atol=1e-14)
    ids[3] = -1
    assert not O.embed_forward(table, ids, scale)[3].any()


def _row_values(x, tok, it):
    logp, entropy, lse, _, _ = O.logprob_forward(x, tok, it)
    return logp, entropy, lse


def test_logprob_matches_torch_and_orders_ties_by_index():
    rng = np.random.default_rng(2)
    x = np.round(rng.normal(size=(5, 37)) * 2) / 2                    # many equal logits
    x[1, 3:9] = -np.inf
    x[2] = -np.inf
    x[3] = -np.inf
    x[3, 30] = 1.5
    tok = np.array([0, 4, 2, 30, -1])
    logp, entropy, lse, top, ids = O.logprob_forward(x, tok, 0.7, 6)
    ref = torch.log_softmax(torch.tensor(x) * 0.7, 1)
    for r in (0, 1, 3):
        np.testing.assert_allclose(logp[r], ref[r, tok[r]], rtol=1e-13)
    assert logp[4] == 0 and logp[2] == -np.inf and lse[2] == -np.inf and entropy[2] == 0
    for r in (0, 1, 4):
        np.testing.assert_allclose(entropy[r], torch.special.entr(ref[r].exp()).sum(), rtol=1e-12)
        np.testing.assert_allclose(lse[r], torch.logsumexp(torch.tensor(x[r]) * 0.7, 0), rtol=1e-13)
        order = sorted(range(37), key=lambda i: (-x[r, i], i))[:6]
        np.testing.assert_array_equal(ids[r], order)
        np.testing.assert_allclose(top[r], ref[r, order], rtol=1e-13)
    assert (ids[2] == -1).all() and list(ids[3]) == [30, -1, -1, -1, -1, -1] and top[3, 0] == 0


def test_logprob_gradient_matches_autograd_and_differences():
    rng = np.random.default_rng(3)
    x, tok, it = rng.normal(size=(4, 9)), np.array([2, -1, 8, 0]), 1.3
    gl, gh, gz = rng.normal(size=(3, 4))
    _, entropy, lse = _row_values(x, tok, it)
    d = O.logprob_backward(x, tok, it, lse, entropy, gl, gh, gz)
    t = torch.tensor(x, requires_grad=True)
    lp = torch.log_softmax(t * it, 1)
    value = (torch.tensor(gh) * -(lp.exp() * lp).sum(1)).sum() + (torch.tensor(gz) * torch.logsumexp(t * it, 1)).sum()
    value = value + sum(gl[r] * lp[r, tok[r]] for r in range(4) if tok[r] >= 0)
    value.backward()
    np.testing.assert_allclose(d, t.grad.numpy(), rtol=1e-10, atol=1e-13)

    def f(x):
        a, b, c = _row_values(x, tok, it)
        return (gl * a + gh * b + gz * c).sum()
    h = 1e-6
    for r in range(4):
        for i in range(9):
            up, down = x.copy(), x.copy()
            up[r, i] += h
            down[r, i] -= h
            assert abs((f(up) - f(down)) / (2 * h) - d[r, i]) < 1e-8


def test_adamw_matches_torch():
    rng = np.random.default_rng(4)
    w = rng.normal(size=50)
    p = torch.nn.Parameter(torch.tensor(w))
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    m, v = np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = rng.normal(size=50)
        p.grad = torch.tensor(g)
        opt.step()
        w, m, v, _ = O.adamw_step(w, g, m, v, 0.01, 0.8, 0.95, 1e-6, t, 0.1)
        np.testing.assert_allclose(w, p.detach().numpy(), rtol=1e-12)


def test_eight_bit_floats():
    codes = np.arange(256, dtype=np.uint8)
    np.testing.assert_array_equal(O.E4M3.astype(np.float32), torch.tensor(codes).view(torch.float8_e4m3fn).float().numpy())
    x = np.random.default_rng(5).normal(size=4000).astype(np.float32) * np.float32(2.0) ** np.random.default_rng(6).integers(-12, 8, 4000)
    x = np.clip(np.concatenate([x, O.E4M3[:127].astype(np.float32), (O.E4M3[:126] + O.E4M3[1:127]).astype(np.float32) / 2]), -448, 448)
    np.testing.assert_array_equal(O._to_e4m3(x), torch.tensor(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert O.E4U4[255] == 1.9375 and O.E4U4[16] == 2.0 ** -14 and (np.diff(O.E4U4) > 0).all()


def test_stochastic_rounding_of_the_second_moment_is_unbiased_and_moves():
    # sqrt(v) decays by 0.05 % a step where the gradient is zero; on average the 8-bit state follows
    n = 4096
    v = np.full(n, 0, np.uint8)
    v[:] = 130
    v[::256] = 255                                        # fixes every block's scale
    vs = np.ones(n // 256, np.float32)
    m, ms = np.zeros(n, np.uint8), np.zeros(n // 256, np.float32)
    live = np.arange(n) % 256 != 0
    start = O.adamw_read8(m, ms, v, vs)[1][live].mean(dtype=np.float64)
    for t in range(1, 41):
        m, ms, v, vs = O.adamw_state8(m, ms, v, vs, np.zeros(n, np.float32), 0.9, 0.999, 77 + t, 0)
    now = O.adamw_read8(m, ms, v, vs)[1][live].mean(dtype=np.float64)
    # each of 4080 elements is off by at most one step of 1/16: three standard errors of the mean are 0.01
    assert abs(now / start - 0.999 ** 40) < 0.01
