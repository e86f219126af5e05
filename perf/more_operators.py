"""Cases for the operators between a model's blocks and its loss: log probabilities straight from the hidden states and the
output head, with their gradients; the join of a block to the residual stream with the norms around it, with its gradient;
dropout.

`run` computes each in plain torch (`own` false) or through the package's entry points (`own` true).
"""
import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # scoring one token of one sequence: the head's weights are read once, nothing else counts
        dict(name="head fwd, one row", op="head_forward", rows=1, vocab=131072, dim=2048, dtype="bf16", temperature=1.0),
        # a small model in float32, no size a multiple of anything, sampled at a temperature
        dict(name="head fwd, f32 odd", op="head_forward", rows=509, vocab=50021, dim=1001, dtype="f32", temperature=0.7),
        # scoring a training batch with a large vocabulary: a gigabyte of logits that is never stored
        dict(name="head fwd, large batch", op="head_forward", rows=4096, vocab=131072, dim=4096, dtype="bf16", temperature=1.0),
        # a short fine-tuning batch under a loss scale
        dict(name="head bwd, short f16", op="head_backward", rows=200, vocab=32000, dim=1024, dtype="f16", temperature=1.0, accumulate=False),
        # a small model in float32 whose table is the head too: the gradient joins what is in the buffer
        dict(name="head bwd, f32 tied", op="head_backward", rows=509, vocab=50021, dim=1000, dtype="f32", temperature=1.25, accumulate=True),
        # a training batch, odd vocabulary
        dict(name="head bwd, bf16 batch", op="head_backward", rows=4096, vocab=100003, dim=2048, dtype="bf16", temperature=1.0, accumulate=False),
        # one decoding step: latency of a single row between two blocks
        dict(name="join fwd, one token", op="join_forward", rows=1, dim=4096, dtype="bf16", stream="bf16", post=True, gate="none", per_gate=1, p=0.0),
        # a training batch of eight sequences, each with a gate vector of its own (conditioning), dropout on the branch
        dict(name="join fwd, gated batch", op="join_forward", rows=16384, dim=4096, dtype="bf16", stream="bf16", post=True, gate="some", per_gate=2048, p=0.1),
        # the same with one learned gate for all tokens and the residual stream in float32
        dict(name="join bwd, bf16 batch", op="join_backward", rows=8192, dim=4096, dtype="bf16", stream="f32", post=True, gate="some", per_gate=8192, p=0.1),
        # a small model in float32, odd sizes, a gate for every token
        dict(name="join bwd, f32 odd", op="join_backward", rows=2047, dim=1001, dtype="f32", stream="f32", post=False, gate="some", per_gate=1, p=0.0),
        # the embeddings of a training batch
        dict(name="dropout, batch", op="dropout", rows=16384, dim=4096, dtype="bf16", p=0.1),
        # a small model's activations, odd sizes
        dict(name="dropout, f32 odd", op="dropout", rows=509, dim=1001, dtype="f32", p=0.35),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["head_forward", "head_backward", "join_forward", "join_backward", "dropout"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op in ("head_forward", "head_backward"):
        vocab, dim = _log(rng, 500, 131072), _log(rng, 16, 4096)
        most = (1 << 40) if op == "head_forward" else (1 << 39)
        rows = _log(rng, 1, max(1, min(8192, most // (vocab * dim), (1 << 29) // vocab)))
        c = dict(op=op, rows=rows, vocab=vocab, dim=dim, dtype=dtype, temperature=round(rng.uniform(0.5, 1.5), 3))
        if op == "head_backward":
            c["accumulate"] = rng.random() < 0.5
        return c
    dim = _log(rng, 16, 8192)
    if op == "dropout":
        return dict(op=op, rows=_log(rng, 1, min(65536, (1 << 26) // dim)), dim=dim, dtype=dtype, p=round(rng.uniform(0.01, 0.6), 3))
    rows = _log(rng, 1, min(65536, (1 << (26 if op == "join_forward" else 25)) // dim))
    return dict(op=op, rows=rows, dim=dim, dtype=dtype, stream=rng.choice(["f32", dtype]), post=rng.random() < 0.5, gate=rng.choice(["none", "some"]),
                per_gate=rng.choice([1, rows, _log(rng, 1, rows)]), p=rng.choice([0.0, round(rng.uniform(0.01, 0.6), 3)]))


def _gates(c):
    return -(-c["rows"] // c["per_gate"]) if c["gate"] == "some" else 0


def work(case):
    c = case
    op, r, d, b = c["op"], c["rows"], c["dim"], BYTES[c["dtype"]]
    if op == "head_forward":
        return {"bytes": (r + c["vocab"]) * d * b + r * 16, "flops": 2 * r * c["vocab"] * d + 5 * r * c["vocab"]}
    if op == "head_backward":
        w = c["vocab"] * d * b
        # the logits again, and one product of their size for each of the two gradients
        return {"bytes": 2 * r * d * b + w * (3 if c["accumulate"] else 2) + r * 24, "flops": 6 * r * c["vocab"] * d + 8 * r * c["vocab"]}
    if op == "dropout":
        return {"bytes": 2 * r * d * b, "flops": r * d}
    s, g = BYTES[c["stream"]], _gates(c) * d * b
    if op == "join_forward":
        return {"bytes": r * d * (2 * s + 2 * b) + g + 2 * d * 4 + 8 * r, "flops": 9 * r * d}
    return {"bytes": r * d * (3 * s + 3 * b) + 2 * g + 4 * d * 4 + 8 * r, "flops": 20 * r * d}


# ------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)                     # noqa: E731
    f = lambda *n: torch.empty(*n, device=DEV)                                     # noqa: E731
    op, r, d, dt = c["op"], c["rows"], c["dim"], DTYPES[c["dtype"]]
    s = {"case": c}
    if op in ("head_forward", "head_backward"):
        v = c["vocab"]
        x = rand(r, d)                                                           # what a norm leaves
        # logits of some units, as a trained head gives
        w = torch.randn(v, d, generator=g, device=DEV, dtype=dt).mul_(1.5 / math.sqrt(d))
        tok = torch.randint(0, v, (r,), generator=g, device=DEV)
        sure = (torch.rand(r, generator=g, device=DEV) < 0.5).float()
        row = w[tok].float()                                                     # half of the rows are confident
        x += row * (sure * 9.0 / row.square().sum(1))[:, None]
        if r > 1:
            tok[torch.rand(r, generator=g, device=DEV) < 0.02] = -1              # padding
        s["hidden"], s["weight"], s["tokens"], s["it"] = x.to(dt), w, tok.to(torch.int32), 1.0 / c["temperature"]
        if op == "head_forward":
            s["logp"], s["entropy"], s["lse"] = f(r), f(r), f(r)
        else:
            each = 256.0 if c["dtype"] == "f16" else 1.0 / r                     # a mean, in f16 with its loss scale
            s["g_logp"] = torch.rand(r, generator=g, device=DEV).add_(0.5).mul_(-each)
            s["g_entropy"] = torch.full((r,), -0.01 * each, device=DEV)
            lse, ent = [], []
            for rows in s["hidden"].split(max(1, (1 << 27) // v)):               # what the forward pass gave
                y = (rows.float() @ w.float().T).double() * s["it"]
                z = y.logsumexp(1)
                p = (y - z[:, None]).exp()
                lse.append(z)
                ent.append(z - (p * y).sum(1))
            s["lse"], s["entropy"] = torch.cat(lse).float(), torch.cat(ent).float()
            s["dhidden"] = torch.empty(r, d, device=DEV, dtype=dt)
            s["dweight"] = torch.randn(v, d, generator=g, device=DEV, dtype=dt).mul_(0.5 * each) if c["accumulate"] else torch.empty(v, d, device=DEV, dtype=dt)
        if own:
            import paper_2003_11666_b200 as pb
            s["scratch"] = torch.empty(pb.head_scratch_bytes(s["hidden"], s["weight"], backward=op == "head_backward"), device=DEV, dtype=torch.uint8)
        return s
    if op == "dropout":
        s["x"], s["out"], s["seed"] = rand(r, d).to(dt), torch.empty(r, d, device=DEV, dtype=dt), int(seed) * 1000003 + 17
        return s
    st = DTYPES[c["stream"]]
    one = lambda: torch.rand(d, generator=g, device=DEV).add_(0.5)                 # noqa: E731
    s["u"], s["seed"] = rand(r, d).mul_(3.0).to(dt), int(seed) * 1000003 + 17
    s["post"], s["pre"] = one() if c["post"] else None, one()
    s["gate"] = rand(_gates(c), d).mul_(0.5).add_(0.3).to(dt) if c["gate"] == "some" else None
    s["rs"] = 0.9
    x = rand(r, d).mul_(2.0).to(st)
    if op == "join_forward":
        s["x"], s["y"], s["h"] = x, torch.empty_like(x), torch.empty(r, d, device=DEV, dtype=dt)
        s["rstd_post"], s["rstd_pre"] = f(r) if c["post"] else None, f(r)
        return s
    # what the forward pass left
    s["y"] = x
    s["rstd_pre"] = (x.double().square().mean(1) + EPS).rsqrt().float()
    s["rstd_post"] = (s["u"].double().square().mean(1) + EPS).rsqrt().float() if c["post"] else None
    s["dy"], s["dh"] = rand(r, d).mul_(0.01).to(st), rand(r, d).mul_(0.02).to(dt)
    s["dx"], s["du"] = torch.empty(r, d, device=DEV, dtype=st), torch.empty(r, d, device=DEV, dtype=dt)
    s["dpost"], s["dpre"] = f(d) if c["post"] else None, f(d)
    s["dgate"] = torch.empty_like(s["gate"]) if s["gate"] is not None else None
    if own:
        import paper_2003_11666_b200 as pb
        s["scratch"] = torch.empty(pb.join_scratch_bytes(r, d, c["per_gate"] if c["gate"] == "some" else 0), device=DEV, dtype=torch.uint8)
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if own:
        import paper_2003_11666_b200 as pb
        if op == "head_forward":
            pb.head_logprob_forward(s["hidden"], s["weight"], s["scratch"], s["tokens"], s["logp"], entropy=s["entropy"], lse=s["lse"],
                                    inv_temperature=s["it"])
            return {k: s[k] for k in ("logp", "entropy", "lse")}
        if op == "head_backward":
            pb.head_logprob_backward(s["hidden"], s["weight"], s["scratch"], s["tokens"], s["lse"], s["dhidden"], s["dweight"], g_logp=s["g_logp"],
                                     g_entropy=s["g_entropy"], entropy=s["entropy"], inv_temperature=s["it"], accumulate=c["accumulate"])
            return {k: s[k] for k in ("dhidden", "dweight")}
        if op == "dropout":
            pb.dropout(s["x"], s["out"], c["p"], s["seed"], offset=3)
            return s["out"]
        per = c["per_gate"] if c["gate"] == "some" else None
        if op == "join_forward":
            pb.join_forward(s["x"], s["u"], s["y"], h=s["h"], pre_weight=s["pre"], post_weight=s["post"], gate=s["gate"], rows_per_gate=per,
                            rstd_pre=s["rstd_pre"], rstd_post=s["rstd_post"], residual_scale=s["rs"], eps=EPS, p=c["p"], seed=s["seed"], offset=3)
            return {k: s[k] for k in ("y", "h", "rstd_pre", "rstd_post")}
        pb.join_backward(s["y"], s["u"], s["dx"], s["du"], s["scratch"], dy=s["dy"], dh=s["dh"], pre_weight=s["pre"], post_weight=s["post"], gate=s["gate"],
                         rows_per_gate=per, rstd_pre=s["rstd_pre"], rstd_post=s["rstd_post"], dpre_weight=s["dpre"], dpost_weight=s["dpost"],
                         dgate=s["dgate"], residual_scale=s["rs"], p=c["p"], seed=s["seed"], offset=3)
        return {k: s[k] for k in ("dx", "du", "dpre", "dpost", "dgate")}
    if op == "head_forward":
        return _head_forward(s["hidden"], s["weight"], s["tokens"], s["it"])
    if op == "head_backward":
        return _head_backward(s["hidden"], s["weight"], s["tokens"], s["lse"], s["entropy"], s["g_logp"], s["g_entropy"], s["it"], s["dweight"],
                              c["accumulate"])
    if op == "dropout":
        x = s["x"].float()
        return (x * _kept(s["seed"], 3, c["p"], x.shape, x.device)).to(s["x"].dtype)
    return _join_forward(s, c) if op == "join_forward" else _join_backward(s, c)


def _head_forward(x, w, tok, it):
    # sums, and the difference of a token's logit and their logarithm, in 64 bits: a confident row's values are near zero
    z = x.float() @ w.float().T
    top = z.amax(1, keepdim=True)
    at = z.gather(1, tok.long().clamp(min=0)[:, None])
    d = (z - top) * it
    e = d.exp()
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    log_z = total.log()
    entropy = log_z - (e * d).sum(1, keepdim=True, dtype=torch.float64) / total
    logp = torch.where(tok[:, None] >= 0, (at - top).double() * it - log_z, 0.0)
    return {"logp": logp[:, 0].float(), "entropy": entropy[:, 0].float(), "lse": (top.double() * it + log_z)[:, 0].float()}


def _head_backward(x, w, tok, lse, entropy, g_logp, g_entropy, it, dweight, accumulate):
    x32, w32 = x.float(), w.float()
    lp = ((x32 @ w32.T).double() * it - lse[:, None]).float()
    p = lp.exp()
    there = (tok >= 0)[:, None]
    at = tok.long().clamp(min=0)[:, None]
    gl = torch.where(there, g_logp[:, None], 0.0)
    h = g_entropy[:, None] * p * (lp + entropy[:, None])
    # the given token: 1 - p without the cancellation
    d = (-gl * p).scatter(1, at, torch.where(there, -gl * torch.expm1(lp.gather(1, at)), -gl * p.gather(1, at)))
    d = (d - h) * it
    dw = d.T @ x32
    if accumulate:
        dw += dweight
    return {"dhidden": (d @ w32).to(x.dtype), "dweight": dweight.copy_(dw)}


def _signed(c):
    return c - (1 << 64) if c >= 1 << 63 else c


def _mix(z):
    """SplitMix64's finaliser of 64-bit integers (torch's int64 products wrap)."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _kept(seed, offset, p, shape, device):
    """What dropout multiplies with: for each element 16 bits of a counter's hash against p."""
    n, gamma = shape[0] * shape[1], 0x9E3779B97F4A7C15
    base = _mix(torch.tensor(_signed((seed + (offset + 1) * gamma) % (1 << 64)), device=device))
    z = _mix((torch.arange(-(-n // 4), device=device) + 1) * _signed(gamma) + base)
    bits = ((z[:, None] >> torch.tensor([0, 16, 32, 48], device=device)) & 0xFFFF).reshape(-1)[:n].reshape(shape)
    drop = int(round(p * 65536))
    return torch.where(bits >= drop, 65536 / (65536 - drop), 0.0).float()


def _by_row(gate, c):
    """The gate's row of every token."""
    return gate.float().repeat_interleave(c["per_gate"], 0)[:c["rows"]]


def _join_forward(s, c):
    x, u = s["x"].float(), s["u"].float()
    rstd_post = None
    b = u
    if c["post"]:
        rstd_post = (u.square().mean(1) + EPS).rsqrt()
        b = u * rstd_post[:, None] * s["post"]
    if s["gate"] is not None:
        b = b * _by_row(s["gate"], c)
    if c["p"] > 0:
        b = b * _kept(s["seed"], 3, c["p"], u.shape, u.device)
    y = x * s["rs"] + b
    rstd_pre = (y.square().mean(1) + EPS).rsqrt()
    h = y * rstd_pre[:, None] * s["pre"]
    return {"y": y.to(s["x"].dtype), "h": h.to(s["u"].dtype), "rstd_pre": rstd_pre, "rstd_post": rstd_post}


def _join_backward(s, c):
    u, dh, r = s["u"].float(), s["dh"].float(), s["rstd_pre"][:, None]
    yn = s["y"].float() * r
    dn = dh * s["pre"]
    dy = s["dy"].float() + (dn - yn * (dn * yn).mean(1, keepdim=True)) * r
    dpre = (dh * yn).sum(0, dtype=torch.float64).float()
    db = dy * _kept(s["seed"], 3, c["p"], u.shape, u.device) if c["p"] > 0 else dy
    un = u * s["rstd_post"][:, None] if c["post"] else u
    n = un * s["post"] if c["post"] else un
    dgate = None
    if s["gate"] is not None:
        groups, per = s["gate"].shape[0], c["per_gate"]
        t = db * n
        if per > 1:
            full = torch.zeros(groups * per, t.shape[1], device=t.device)
            full[:c["rows"]] = t
            t = full.view(groups, per, -1).sum(1, dtype=torch.float64)
        dgate = t.to(s["gate"].dtype)
        db = db * _by_row(s["gate"], c)
    du, dpost = db, None
    if c["post"]:
        dpost = (db * un).sum(0, dtype=torch.float64).float()
        dn = db * s["post"]
        du = (dn - un * (dn * un).mean(1, keepdim=True)) * s["rstd_post"][:, None]
    return {"dx": (dy * s["rs"]).to(s["y"].dtype), "du": du.to(s["u"].dtype), "dpre": dpre, "dpost": dpost, "dgate": dgate}


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c, op, r, d = case, case["op"], case["rows"], case["dim"]
    f = torch.float64
    if op == "dropout":
        return s["x"].to(f) * _mask_again(s["seed"], 3, c["p"], r, d)
    if op in ("head_forward", "head_backward"):
        v = c["vocab"]
        w = s["weight"].to(f)
        at_once = max(1, (1 << 28) // v)
        got = [[], [], []]
        dw = torch.zeros(v, d, dtype=f, device=DEV) if op == "head_backward" else None
        for k in range(0, r, at_once):
            at = slice(k, min(r, k + at_once))
            x, tok = s["hidden"][at].to(f), s["tokens"][at].long()
            z = torch.mm(x, w.T).mul_(s["it"])
            rows = torch.arange(len(tok), device=DEV)
            if op == "head_forward":
                lp = torch.log_softmax(z, 1)
                got[0].append(torch.where(tok >= 0, lp[rows, tok.clamp(min=0)], 0.0))
                got[1].append(torch.special.entr(lp.exp()).sum(1))
                got[2].append(torch.logsumexp(z, 1))
                continue
            lp = z - s["lse"][at, None].to(f)
            p = lp.exp()
            gl = s["g_logp"][at].to(f) * (tok >= 0)
            dz = s["g_entropy"][at, None].to(f) * (torch.special.entr(p) - p * s["entropy"][at, None].to(f)) - gl[:, None] * p
            dz[rows, tok.clamp(min=0)] += gl
            dz *= s["it"]
            got[0].append(torch.mm(dz, w))
            dw.addmm_(dz.T, x)
        if op == "head_forward":
            return dict(zip(("logp", "entropy", "lse"), (torch.cat(x) for x in got)))
        if c["accumulate"]:
            dw += s["dweight"]
        return {"dhidden": torch.cat(got[0]), "dweight": dw}
    u = s["u"].to(f)
    gate = s["gate"].to(f)[torch.arange(r, device=DEV) // c["per_gate"]] if s["gate"] is not None else torch.ones(1, 1, dtype=f, device=DEV)
    keep = _mask_again(s["seed"], 3, c["p"], r, d) if c["p"] > 0 else torch.ones(1, 1, dtype=f, device=DEV)
    post = s["post"].to(f) if c["post"] else torch.ones(d, dtype=f, device=DEV)
    if op == "join_forward":
        rp = 1 / torch.sqrt(EPS + u.pow(2).sum(1) / d) if c["post"] else None
        n = torch.einsum("td,t,d->td", u, rp, post) if c["post"] else u
        y = s["rs"] * s["x"].to(f) + keep * gate * n
        rr = 1 / torch.sqrt(EPS + y.pow(2).sum(1) / d)
        return {"y": y, "h": torch.einsum("td,t,d->td", y, rr, s["pre"].to(f)), "rstd_pre": rr, "rstd_post": rp}
    y, dh, rr = s["y"].to(f), s["dh"].to(f), s["rstd_pre"].to(f)
    wd = dh * s["pre"].to(f)
    dy = s["dy"].to(f) + rr[:, None] * wd - (rr ** 3 / d * (wd * y).sum(1))[:, None] * y
    rp = s["rstd_post"].to(f) if c["post"] else torch.ones(r, dtype=f, device=DEV)
    db = dy * keep
    un = u * rp[:, None]
    dgate = None
    if s["gate"] is not None:
        dgate = torch.zeros(s["gate"].shape, dtype=f, device=DEV).index_add_(0, torch.arange(r, device=DEV) // c["per_gate"], db * un * post)
    dn = db * gate
    du = dn
    if c["post"]:
        du = rp[:, None] * dn * post - (rp ** 3 / d * (dn * post * u).sum(1))[:, None] * u
    return {"dx": s["rs"] * dy, "du": du, "dpre": torch.einsum("td,td,t->d", dh, y, rr), "dpost": (dn * un).sum(0) if c["post"] else None, "dgate": dgate}


def _mask_again(seed, offset, p, rows, cols):
    """Dropout's factors from unsigned 64-bit arithmetic in numpy."""
    import numpy as np
    gamma, a, b = np.uint64(0x9E3779B97F4A7C15), np.uint64(0xBF58476D1CE4E5B9), np.uint64(0x94D049BB133111EB)

    def hashed(z):
        z = (z ^ (z >> np.uint64(30))) * a
        z = (z ^ (z >> np.uint64(27))) * b
        return z ^ (z >> np.uint64(31))

    with np.errstate(over="ignore"):
        start = hashed(np.array([seed % (1 << 64)], np.uint64) + np.array([offset + 1], np.uint64) * gamma)
        quads = hashed(start + np.arange(1, (rows * cols + 3) // 4 + 1, dtype=np.uint64) * gamma)
    bits = quads.astype("<u8").view("<u2")[:rows * cols].reshape(rows, cols)
    drop = int(round(p * 65536))
    return torch.from_numpy(np.where(bits >= drop, 65536.0 / (65536 - drop), 0.0)).to(DEV)
