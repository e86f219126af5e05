"""Plain float64 forms of the operators between a model's blocks and its loss, on torch tensors of any device: log
probabilities of hidden states under a head, the join of a block to the residual stream, dropout, and their gradients.

Beside each value `*_error` gives a bound on what float32 arithmetic may be off by; see there.
"""
import numpy as np
import torch

U = 2.0 ** -24


# ---------------------------------------------------------------- which elements dropout keeps
def keep(seed, offset, p, rows, dim):
    """Factors of dropout: SplitMix64 in Python's and numpy's unsigned integers."""
    gamma, mask = 0x9E3779B97F4A7C15, (1 << 64) - 1

    def finish(z):
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & mask
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & mask
        return z ^ (z >> 31)
    base = finish((seed + (offset + 1) * gamma) & mask)
    with np.errstate(over="ignore"):
        z = np.uint64(base) + (np.arange((rows * dim + 3) // 4, dtype=np.uint64) + np.uint64(1)) * np.uint64(gamma)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    bits = np.stack([(z >> np.uint64(16 * k)) & np.uint64(0xFFFF) for k in range(4)], 1).reshape(-1)[:rows * dim].reshape(rows, dim)
    drop = int(round(p * 65536))
    return torch.from_numpy(np.where(bits.astype(np.int64) >= drop, 65536.0 / (65536 - drop), 0.0))


# ---------------------------------------------------------------- head
def head_forward(hidden, weight, tokens, it):
    """logp (0 without a token), entropy, lse, and the logits times `it`."""
    z = hidden.double() @ weight.double().T * it
    lse = z.logsumexp(1)
    p = (z - lse[:, None]).exp()
    entropy = lse - (p * z).sum(1)
    logp = None
    if tokens is not None:
        ok = (tokens >= 0) & (tokens < weight.shape[0])
        logp = torch.where(ok, z.gather(1, torch.where(ok, tokens, 0).long()[:, None])[:, 0] - lse, 0.0)
    return logp, entropy, lse, z


def head_logit_error(hidden, weight, it):
    """Bound on a logit's error, [rows, vocab].  With S the sum of the magnitudes of its terms: the tensor core adds 16 products
    at a time to its accumulator and each time drops less than 2^-22 of what it holds (bits behind the float32 accumulator's last,
    and of aligned products).  A float32 product is at most 48 such steps (three terms of 256 columns, or six of 128) before float32
    registers take over; 16-bit ones are summed through at most 4096 columns (256 steps) by themselves.  What it holds grows with the steps, so
    that half of them count, and four more for the products' own alignment.  Adding the parts costs U of each, a float32 operand in two
    planes U of it, or 2^-39 of the largest among the 32 rows that share a scale (for hidden rows, of their own), the term left out U, the scale by a float32 inv_temperature 2 U."""
    f32, n = hidden.dtype is torch.float32, hidden.shape[1]
    h, w = hidden.double().abs(), weight.double().abs()
    s = h @ w.T * it
    if not f32:
        return s * ((min(n, 4096) / 32 + 4) * 2.0 ** -22 + (-(-n // 2048) + 5) * U)
    floor = 2.0 ** -38 * it * (h.amax(1)[:, None] * w.sum(1)[None] + h.sum(1)[:, None] * w.max())
    return s * (28 * 2.0 ** -22 + (-(-n // 256) + 5) * U) + floor


def head_forward_error(hidden, weight, tokens, it):
    """Bounds for logp, entropy and lse.  A shift e of the logits moves lse by e at most, logp by 2 e, the entropy by
    e * 2 entropy; exponentials and sums are good to 2^-20 of the sum (2^-22 each, 2 + 2^-24 per 32 joined parts)."""
    logp, entropy, lse, z = head_forward(hidden, weight, tokens, it)
    e = head_logit_error(hidden, weight, it).max(1).values
    near = (z - lse[:, None]).abs().amax(1)                        # numbers that are rounded before they are exponents
    base = 2.0 ** -20 + 4 * U * (near + z.abs().amax(1))
    return 2 * e + base + 2 * U * (0 if logp is None else logp.abs()), 2 * e * entropy + base * (1 + 2 * entropy), e + base + 2 * U * lse.abs()


def head_backward(hidden, weight, tokens, it, lse, entropy=None, g_logp=None, g_entropy=None, g_lse=None):
    """d (gradient with respect to the logits), dhidden, dweight, from the lse (and entropy) given."""
    z = hidden.double() @ weight.double().T * it
    lp = z - lse.double()[:, None]
    p = lp.exp()
    d = torch.zeros_like(z)
    if g_logp is not None:
        ok = (tokens >= 0) & (tokens < weight.shape[0])
        gl = torch.where(ok, g_logp, 0.0).double()[:, None]
        d -= gl * p
        d.scatter_add_(1, torch.where(ok, tokens, 0).long()[:, None], gl)
    if g_entropy is not None:
        d -= g_entropy.double()[:, None] * p * (lp + entropy.double()[:, None])
    if g_lse is not None:
        d += g_lse.double()[:, None] * p
    d *= it
    return d, d @ weight.double(), d.T @ hidden.double(), lp


def head_backward_error(hidden, weight, tokens, it, lse, entropy, g_logp, g_entropy, g_lse, half, store):
    """Bounds for dhidden and dweight (before what an accumulated dweight adds).  `half`: the relative rounding of d, which is held
    in the operands' type (0 stands for float32's planes, 2^-24); float16 also has a smallest number, 2^-25 of a scale at which
    the largest coefficient of d is 2^13 or more.  `store`: the rounding of the outputs."""
    d, dh, dw, lp = head_backward(hidden, weight, tokens, it, lse, entropy, g_logp, g_entropy, g_lse)
    zero = torch.zeros_like(lse, dtype=torch.float64)
    c = lambda g: zero if g is None else g.double().abs()         # noqa: E731
    a, ge, gz = c(g_logp) * it, c(g_entropy) * it, c(g_lse) * it
    h = zero if entropy is None else entropy.double().abs()
    size = (a + gz + ge * h)[:, None] + ge[:, None] * lp.abs()      # |d| / p, and what its sum is made of
    off = head_logit_error(hidden, weight, it) + 4 * U * (lp.abs() + (lp + lse.double()[:, None]).abs() + lse.double().abs()[:, None]) + 2.0 ** -21
    ed = d.abs() * (half or U) + lp.exp() * (size + ge[:, None]) * off + 8 * U * lp.exp() * size
    if half == 2.0 ** -11:
        ed += 2.0 ** -38 * 2 * (a * 2 + gz + ge * h + ge).max()
    w, x = weight.double().abs(), hidden.double().abs()
    # the products' own sums: 16 products at a time, over the whole length for 16-bit operands
    long = lambda n: (n / 16 + 1) * 2.0 ** -22 if half else 28 * 2.0 ** -22 + (n / 128 + 5) * U      # noqa: E731
    # float32: dhidden's planes of d hold 2^-25 of a scale at which the row's largest coefficient is 2^13 or more, and the largest weight 2^14
    floor = 0 if half else 2.0 ** -37 * weight.shape[0] * w.max() * (2 * a + gz + ge * h + ge)[:, None]
    eh = floor + ed @ w + (d.abs() @ w) * (long(weight.shape[0]) + 8 * U) + store * dh.abs()
    ew = ed.T @ x + (d.abs().T @ x) * (long(hidden.shape[0]) + 4 * U) + store * dw.abs()
    return eh, ew


# ---------------------------------------------------------------- join
def join_forward(x, u, gate, per, post, pre, rs, eps, factor):
    """y, h, rstd_post, rstd_pre."""
    x, u = x.double(), u.double()
    rp = None
    b = u
    if post is not None:
        rp = (u.square().mean(1) + eps).rsqrt()
        b = u * rp[:, None] * post.double()
    if gate is not None:
        b = b * gate.double()[torch.arange(x.shape[0], device=x.device) // per]
    y = rs * x + (b if factor is None else b * factor)
    rr = (y.square().mean(1) + eps).rsqrt()
    return y, None if pre is None else y * rr[:, None] * pre.double(), rp, rr


def join_backward(y, u, dy, dh, gate, per, post, pre, rp, rr, rs, factor):
    """dict of dx, du, dgate, dpost, dpre, each with its bound for float32 arithmetic before it is stored ("e_" + name).
    A mean of dim products costs 34 U of the mean of their magnitudes (16 columns per thread, up to 10 levels of
    threads, the products, the factor 1 / dim); a sum over n rows (n + 4) U of the sum of the magnitudes; a product U."""
    rows, dim = u.shape
    u = u.double()
    dy_ = torch.zeros(rows, dim, dtype=torch.float64, device=u.device) if dy is None else dy.double()
    out, e = {}, 2 * U * dy_.abs()
    g = dy_
    if dh is not None:
        yn, w = y.double() * rr.double()[:, None], dh.double() * pre.double()
        m = (w * yn).mean(1, keepdim=True)
        g = dy_ + rr.double()[:, None] * (w - m * yn)
        e = e + rr.double()[:, None] * ((34 * (w * yn).abs().mean(1, keepdim=True) + 4 * m.abs()) * yn.abs() + 4 * w.abs()) * U + 2 * U * g.abs()
        out["dpre"] = (dh.double() * yn).sum(0)
        out["e_dpre"] = (rows + 4) * U * (dh.double() * yn).abs().sum(0)
    out["dx"], out["e_dx"] = rs * g, abs(rs) * e + 2 * U * (rs * g).abs()
    if factor is not None:
        g, e = g * factor, e * factor + U * (g * factor).abs()
    un = u if rp is None else u * rp.double()[:, None]
    n = un if post is None else un * post.double()
    if gate is not None:
        row = torch.arange(rows, device=u.device) // per
        z = torch.zeros(gate.shape, dtype=torch.float64, device=u.device)
        out["dgate"] = z.index_add(0, row, g * n)
        out["e_dgate"] = z.index_add(0, row, e * n.abs()) + (min(per, rows) + 6) * U * z.index_add(0, row, (g * n).abs())
        k = gate.double()[row]
        g, e = g * k, e * k.abs() + U * (g * k).abs()
    if post is not None:
        out["dpost"] = (g * un).sum(0)
        out["e_dpost"] = (e * un.abs()).sum(0) + (rows + 6) * U * (g * un).abs().sum(0)
        w = g * post.double()
        ew = e * post.double().abs() + U * w.abs()
        m = (w * un).mean(1, keepdim=True)
        em = 34 * U * (w * un).abs().mean(1, keepdim=True) + (ew * un.abs()).mean(1, keepdim=True)
        r = rp.double()[:, None]
        g = r * (w - m * un)
        e = r * (ew + em * un.abs() + 4 * U * (w.abs() + (m * un).abs()))
    out["du"], out["e_du"] = g, e + 2 * U * g.abs()
    return out
