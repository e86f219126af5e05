"""Token operators for the CPU oracle (test infrastructure; float64): embedding lookup and
its gradient, log probabilities of given tokens with entropy and alternatives and their
gradient, and the AdamW step.

Written from the definitions, row by row and without blocking.  The 8-bit AdamW state is
defined on float32 moments with every operation rounded, so `adamw_state8` follows those
roundings with numpy's float32; everything else is float64.
"""
import numpy as np


# ---------------------------------------------------------------- embedding
def embed_forward(table, ids, scale):
    out = np.zeros((len(ids), table.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < table.shape[0]:
            out[t] = scale * table[v]
    return out


def embed_backward(dout, ids, vocab, scale, padding=-1, start=None):
    """dtable, added to `start` if given."""
    d = np.zeros((vocab, dout.shape[1])) if start is None else np.array(start, dtype=np.float64)
    for t, v in enumerate(ids):
        if 0 <= v < vocab and v != padding:
            d[v] += scale * dout[t]
    return d


# ---------------------------------------------------------------- log probabilities
def logprob_forward(x, tokens, it, k=0):
    """(logp, entropy, lse, top_logp, top_ids) of rows of logits; see include/pb.h for rows without
    a finite logit and rows with NaN or +inf."""
    rows, vocab = x.shape
    logp, entropy, lse = np.zeros(rows), np.zeros(rows), np.zeros(rows)
    top_logp, top_ids = np.full((rows, k), -np.inf), np.full((rows, k), -1, dtype=np.int32)
    for r in range(rows):
        v = x[r].astype(np.float64)
        tok = int(tokens[r]) if tokens is not None and 0 <= tokens[r] < vocab else None
        if np.isnan(v).any() or (v == np.inf).any():
            entropy[r] = lse[r] = top_logp[r] = np.nan
            logp[r] = np.nan if tok is not None else 0.0
            continue
        m = v.max()
        if m == -np.inf:
            logp[r] = -np.inf if tok is not None else 0.0
            lse[r] = -np.inf
            continue
        d = (v - m) * it
        e = np.exp(d)
        first = int(np.argmax(v))
        rest = e.sum() - e[first] if vocab < 2 else np.delete(e, first).sum()
        log_z = np.log1p(rest)
        live = e > 0
        lse[r] = m * it + log_z
        entropy[r] = log_z - (e[live] * d[live]).sum() / (1.0 + rest)
        if tok is not None:
            logp[r] = d[tok] - log_z
        order = np.lexsort((np.arange(vocab), -v))[:k]
        for q, i in enumerate(order):
            if v[i] > -np.inf:
                top_ids[r, q], top_logp[r, q] = i, d[i] - log_z
    return logp, entropy, lse, top_logp, top_ids


def logprob_backward(x, tokens, it, lse, entropy=None, g_logp=None, g_entropy=None, g_lse=None):
    d = np.zeros(x.shape)
    for r in range(x.shape[0]):
        if lse[r] == -np.inf:
            continue
        lp = x[r].astype(np.float64) * it - float(lse[r])
        p = np.exp(lp)
        if g_logp is not None and 0 <= tokens[r] < x.shape[1]:
            one = np.zeros_like(p)
            one[int(tokens[r])] = 1.0
            d[r] += g_logp[r] * (one - p)
        if g_entropy is not None:
            d[r] -= g_entropy[r] * p * (np.where(p > 0, lp, 0.0) + entropy[r])
        if g_lse is not None:
            d[r] += g_lse[r] * p
        d[r] *= it
    return d


# ---------------------------------------------------------------- AdamW
def adamw_step(w, g, m, v, lr, beta1, beta2, eps, step, decay):
    """(w, m, v, u): decoupled weight decay, bias-corrected moments, u the update's direction."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    u = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return w - lr * decay * w - lr * u, m, v, u


BLOCK = 256
E4M3 = np.array([(-1.0 if c & 128 else 1.0) * ((c & 7) / 8 * 2.0 ** -6 if not c & 120 else (1 + (c & 7) / 8) * 2.0 ** (((c >> 3) & 15) - 7))
                 for c in range(256)])
E4M3[[127, 255]] = np.nan
E4U4 = np.array([0.0] + [2.0 ** (c // 16 - 15) * (1 + (c % 16) / 16) for c in range(1, 256)])


def _to_e4m3(x):
    """Codes of the nearest value, the even code between two; |x| up to 448."""
    values = E4M3[:127]
    a = np.abs(x.astype(np.float64))
    lo = np.clip(np.searchsorted(values, a, side="right") - 1, 0, 126)
    hi = np.minimum(lo + 1, 126)
    up = a - values[lo] > values[hi] - a
    tie = (a - values[lo] == values[hi] - a) & (lo != hi)
    code = np.where(up | (tie & (lo % 2 == 1)), hi, lo)
    return (code + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def random16(seed, tensor, i):
    """The 16 random bits of element i: SplitMix64 (Steele, Lea & Flood 2014), one draw for four elements."""
    mask = (1 << 64) - 1
    z = (seed * 0xD1342543DE82EF95 + tensor * 0xA0761D6478BD642F + (i // 4 + 1) * 0x9E3779B97F4A7C15) & mask
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & mask
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & mask
    z ^= z >> 31
    return (z >> (16 * (i % 4))) & 0xFFFF


def adamw_read8(m, ms, v, vs):
    """The float32 moments of an 8-bit state."""
    f, n = np.float32, len(m)
    k = np.arange(n) // BLOCK
    with np.errstate(invalid="ignore"):
        r = E4U4[v].astype(f) * vs[k]
        return E4M3[m].astype(f) * ms[k], r * r


def adamw_state8(m, ms, v, vs, g, beta1, beta2, seed, tensor):
    """New (m codes, m scales, v codes, v scales) from the float32 gradient g; `seed` is the call's seed + step."""
    f, n = np.float32, len(g)
    blocks = -(-n // BLOCK)
    with np.errstate(all="ignore"):
        m32, v32 = adamw_read8(m, ms, v, vs)
        m32 = f(beta1) * m32 + f(1 - beta1) * g
        v32 = f(beta2) * v32 + (f(1 - beta2) * g) * g
        r32 = np.sqrt(v32)
        mc, vc = np.zeros(n, np.uint8), np.zeros(n, np.uint8)
        mo, vo = np.zeros(blocks, f), np.zeros(blocks, f)
        for b in range(blocks):
            at = slice(b * BLOCK, min(n, (b + 1) * BLOCK))
            mb, rb = m32[at], r32[at]
            ma, ra = np.abs(mb).max(), rb.max()
            if not np.isfinite(ma):
                mo[b] = np.nan
            elif ma >= f(2.0 ** -100):
                mc[at] = _to_e4m3(mb * (f(448) / ma))
                mo[b] = ma * (f(1) / f(448))
            if not np.isfinite(ra):
                vo[b] = np.nan
            elif ra > 0:
                x = rb * (f(1.9375) / ra)
                vo[b] = ra / f(1.9375)
                for q, i in enumerate(range(at.start, at.stop)):
                    code = ((int(x[q].view(np.uint32)) + (random16(seed, tensor, i) << 3)) >> 19) - 1792
                    vc[i] = min(max(code, 1), 255) if rb[q] > 0 else 0
    return mc, mo, vc, vo
