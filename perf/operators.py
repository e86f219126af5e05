"""Cases for the token operators: embedding and its gradient, log probabilities of given tokens and
their gradient, AdamW over many tensors with states in 32 or 8 bits.

`run` computes each in plain torch (`own` false) or through the package's entry points (`own` true).
"""
import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "int32": 4, "int64": 8}
BLOCK = 256                       # elements of an 8-bit state that share a scale
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.01


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decoding step of one sequence: latency of a single row
        dict(name="embed fwd, one token", op="embed_forward", tokens=1, vocab=32000, dim=2048, dtype="bf16", ids="int64"),
        # a training batch of long sequences, input scaled by sqrt(dim)
        dict(name="embed fwd, long batch", op="embed_forward", tokens=16384, vocab=131072, dim=4096, dtype="bf16", ids="int64"),
        # a small model's batch, odd sizes, gradient of the whole table written
        dict(name="embed bwd, dense f32", op="embed_backward", tokens=2047, vocab=50021, dim=1000, dtype="f32", ids="int32", grad="f32", accumulate=False),
        # tied table: the gradient joins the head's, already in the buffer; frequent tokens repeat a thousand times
        dict(name="embed bwd, tied bf16", op="embed_backward", tokens=65536, vocab=131072, dim=2048, dtype="bf16", ids="int64", grad="f32", accumulate=True),
        # scoring one decoding step with 20 alternatives
        dict(name="logprob fwd, one row", op="logprob_forward", rows=1, vocab=131072, dtype="bf16", top=20, temperature=1.0),
        # a serving batch at a temperature
        dict(name="logprob fwd, serving batch", op="logprob_forward", rows=200, vocab=32000, dtype="f32", top=5, temperature=0.7),
        # scoring a training batch: rows of an odd length, so that no two start on the same alignment
        dict(name="logprob fwd, long odd rows", op="logprob_forward", rows=4096, vocab=100003, dtype="bf16", top=8, temperature=1.0),
        # training with an entropy bonus, odd rows in float32
        dict(name="logprob bwd, f32 odd", op="logprob_backward", rows=509, vocab=50021, dtype="f32", temperature=1.25),
        # training batch in bf16
        dict(name="logprob bwd, bf16 batch", op="logprob_backward", rows=4096, vocab=65536, dtype="bf16", temperature=1.0),
        # the four-stage MLP of the benchmark: eight small tensors, one after the other in one flat vector
        dict(name="adamw, small mlp", op="adamw", shapes="mlp", depth=4, width=256, first=784, last=10, bits=32, grad="f32", forward="none", horizon=0.0),
        # the sixteen-stage MLP of the benchmark with bf16 forward weights beside float32 masters
        dict(name="adamw, deep mlp", op="adamw", shapes="mlp", depth=16, width=2048, first=2048, last=10, bits=32, grad="f32", forward="bf16", horizon=0.0),
        # blocks of six tensors each, 8-bit states, bf16 gradients, forward weights predicted 6 steps ahead
        dict(name="adamw, 8-bit blocks", op="adamw", shapes="blocks", depth=12, width=1024, first=0, last=0, bits=8, grad="bf16", forward="bf16", horizon=6.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed_forward", "embed_backward", "logprob_forward", "logprob_backward", "adamw"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op == "embed_forward":
        dim = _log(rng, 16, 8192)
        return dict(op=op, tokens=_log(rng, 1, min(65536, (1 << 27) // dim)), vocab=_log(rng, 1000, min(200000, (1 << 29) // dim)), dim=dim,
                    dtype=dtype, ids=rng.choice(["int32", "int64"]))
    if op == "embed_backward":
        dim = _log(rng, 16, 4096)
        return dict(op=op, tokens=_log(rng, 1, min(65536, (1 << 26) // dim)), vocab=_log(rng, 1000, min(200000, (1 << 28) // dim)), dim=dim,
                    dtype=dtype, ids=rng.choice(["int32", "int64"]), grad=rng.choice(["f32", dtype]), accumulate=rng.random() < 0.5)
    if op == "logprob_forward":
        vocab = _log(rng, 500, 200000)
        return dict(op=op, rows=_log(rng, 1, min(8192, (1 << 27) // vocab)), vocab=vocab, dtype=dtype, top=rng.randint(0, 32),
                    temperature=round(rng.uniform(0.5, 1.5), 3))
    if op == "logprob_backward":
        vocab = _log(rng, 500, 200000)
        return dict(op=op, rows=_log(rng, 1, min(8192, (1 << 27) // vocab)), vocab=vocab, dtype=dtype,
                    temperature=round(rng.uniform(0.5, 1.5), 3))
    width = _log(rng, 32, 1600)
    return dict(op=op, shapes=rng.choice(["mlp", "blocks"]), depth=rng.randint(1, 6), width=width, first=_log(rng, 8, 2000), last=_log(rng, 2, 1000),
                bits=rng.choice([32, 8]), grad=dtype, forward=rng.choice(["none", "f32", "bf16", "f16"]), horizon=float(rng.randint(0, 12)))


def _sizes(c):
    """Elements of each tensor of an AdamW case."""
    w = c["width"]
    if c["shapes"] == "mlp":
        dims = [c["first"]] + [w] * (c["depth"] - 1) + [c["last"]]
        return [n for a, b in zip(dims[:-1], dims[1:]) for n in (a * b, b)]
    return [n for _ in range(c["depth"]) for n in (w, 3 * w * w + 3 * w, w * w, w, 4 * w * w, 4 * w * w)]


def work(case):
    c = case
    op = c["op"]
    if op in ("embed_forward", "embed_backward"):
        t, v, d, b = c["tokens"], c["vocab"], c["dim"], BYTES[c["dtype"]]
        distinct = _distinct(t, v)
        if op == "embed_forward":
            return {"bytes": t * BYTES[c["ids"]] + distinct * d * b + t * d * b, "flops": t * d}
        out = BYTES[c["grad"]] * d * (2 * distinct if c["accumulate"] else v)
        return {"bytes": t * BYTES[c["ids"]] + t * d * b + out, "flops": t * d}
    if op == "logprob_forward":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * BYTES[c["dtype"]] + c["rows"] * (4 + 12 + 8 * c["top"]), "flops": 5 * n}
    if op == "logprob_backward":
        n = c["rows"] * c["vocab"]
        return {"bytes": 2 * n * BYTES[c["dtype"]] + c["rows"] * 20, "flops": 8 * n}
    n = sum(_sizes(c))
    b = 8 + BYTES[c["grad"]] + (BYTES[c["forward"]] if c["forward"] != "none" else 0)
    # 8-bit: both codes read and written, and both moments given back as the float32 values they stand for
    return {"bytes": n * (b + 16 if c["bits"] == 32 else b + 4 + 16 / BLOCK + 8), "flops": 15 * n}


def _distinct(tokens, vocab):
    """Expected number of different ids among floor(vocab * u^3), u uniform, the table taken in 1024 slices."""
    total, rows = 0.0, max(1.0, vocab / 1024)
    for k in range(1024):
        share = ((k + 1) / 1024) ** (1 / 3) - (k / 1024) ** (1 / 3)
        total += vocab / 1024 * -math.expm1(tokens * math.log1p(-min(0.999999, share / rows)))
    return min(tokens, max(1.0, total))


# ------------------------------------------------------------------------------------------ inputs
def _tokens(g, n, vocab, dtype, none=0.01):
    """Ids as text has them: a few very frequent, a long tail, one in a hundred no token (-1)."""
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    ids = (u ** 3 * vocab).long().clamp_(0, vocab - 1)
    if n > 1:
        ids[torch.rand(n, generator=g, device=DEV) < none] = -1
    return ids.to(torch.int32 if dtype == "int32" else torch.int64)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)                     # noqa: E731
    s = {"case": c}
    op = c["op"]
    if op in ("embed_forward", "embed_backward"):
        t, v, d, dt = c["tokens"], c["vocab"], c["dim"], DTYPES[c["dtype"]]
        s["ids"] = _tokens(g, t, v, c["ids"])
        s["scale"] = math.sqrt(d)
        if op == "embed_forward":
            s["table"] = torch.randn(v, d, generator=g, device=DEV, dtype=dt).mul_(0.02)
            s["out"] = torch.empty(t, d, device=DEV, dtype=dt)
        else:
            s["dout"] = rand(t, d).mul_(0.01).to(dt)
            s["pad"] = v - 1
            gd = DTYPES[c["grad"]]
            s["dtable"] = torch.randn(v, d, generator=g, device=DEV, dtype=gd).mul_(0.01) if c["accumulate"] else torch.empty(v, d, device=DEV, dtype=gd)
            if own:
                import paper_2003_11666_b200 as pb
                s["scratch"] = torch.empty(pb.embed_scratch_bytes(t, v, d), device=DEV, dtype=torch.uint8)
    elif op in ("logprob_forward", "logprob_backward"):
        r, v = c["rows"], c["vocab"]
        x = torch.randn(r, v, generator=g, device=DEV, dtype=DTYPES[c["dtype"]]).mul_(2.5)
        tok = torch.randint(0, v, (r,), generator=g, device=DEV)
        sure = torch.arange(r, device=DEV)[torch.rand(r, generator=g, device=DEV) < 0.5]
        x[sure, tok[sure]] += 12.0                                               # half of the rows are confident
        if v > 1000:
            x[:, 100:110] = -math.inf                                            # tokens that are never allowed
        if r > 1:
            tok[torch.rand(r, generator=g, device=DEV) < 0.02] = -1              # padding
        s["logits"], s["tokens"], s["it"] = x, tok.to(torch.int32), 1.0 / c["temperature"]
        f = lambda *n: torch.empty(*n, device=DEV)                               # noqa: E731
        if op == "logprob_forward":
            s["logp"], s["entropy"], s["lse"] = f(r), f(r), f(r)
            s["top_logp"] = f(r, c["top"])
            s["top_ids"] = torch.empty(r, c["top"], device=DEV, dtype=torch.int32)
        else:
            each = 256.0 if c["dtype"] == "f16" else 1.0 / r                     # a mean, in f16 with its loss scale
            s["g_logp"] = torch.rand(r, generator=g, device=DEV).add_(0.5).mul_(-each)
            s["g_entropy"] = torch.full((r,), -0.01 * each, device=DEV)
            lse, ent = [], []
            for rows in x.split(max(1, (1 << 27) // v)):                         # what the forward pass gave
                y = rows.double() * s["it"]
                z = y.logsumexp(1)
                p = (y - z[:, None]).exp()
                lse.append(z)
                ent.append(z - (p * torch.where(p > 0, y, 0.0)).sum(1))
            s["lse"], s["entropy"] = torch.cat(lse).float(), torch.cat(ent).float()
            s["dlogits"] = torch.empty_like(x)
    else:
        sizes, eight = _sizes(c), c["bits"] == 8
        room = [-(-n // BLOCK) * BLOCK if eight or c["shapes"] == "blocks" else n for n in sizes]
        at = [sum(room[:k]) for k in range(len(room))]
        total = sum(room)
        view = lambda flat: [flat[a:a + n] for a, n in zip(at, sizes)]           # noqa: E731
        s["sizes"], s["step"], s["seed"] = sizes, 9, int(seed) & 0xFFFF
        s["w"] = rand(total).mul_(0.02)
        s["grad"] = torch.empty(total, device=DEV, dtype=DTYPES[c["grad"]])
        s["grad"].copy_(rand(total).mul_(torch.rand(total, generator=g, device=DEV).mul_(-9).exp_()))
        s["scale"] = torch.full((), 0.5, device=DEV)                             # what clipping left of the gradient
        m, r = rand(total).mul_(0.1), torch.rand(total, generator=g, device=DEV).add_(0.01).mul_(0.3)
        if eight:
            for a, n, k in zip(at, sizes, room):
                m[a + n:a + k] = 0
                r[a + n:a + k] = 0
            mb, rb = m.view(-1, BLOCK), r.view(-1, BLOCK)
            s["m_scale"], s["v_scale"] = mb.abs().amax(1) / 448.0, rb.amax(1) / 1.9375
            s["m"] = (mb / s["m_scale"][:, None]).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).reshape(-1)
            code = ((rb / s["v_scale"][:, None]).view(torch.int32) >> 19) - 1792
            s["v"] = torch.where(rb > 0, code.clamp_(1, 255), 0).to(torch.uint8).reshape(-1)
            s["m_read"], s["v_read"] = torch.empty(total, device=DEV), torch.empty(total, device=DEV)
        else:
            s["m"], s["v"] = m, r.square()
        s["forward"] = torch.zeros(total, device=DEV, dtype=DTYPES[c["forward"]]) if c["forward"] != "none" else None
        s["lists"] = {k: view(s[k]) for k in ("w", "grad", "m", "v")}
        if s["forward"] is not None:
            s["lists"]["forward"] = view(s["forward"])
        if eight:
            cut = lambda flat: [flat[a // BLOCK:(a + k) // BLOCK] for a, k in zip(at, room)]   # noqa: E731
            s["lists"]["m_scale"], s["lists"]["v_scale"] = cut(s["m_scale"]), cut(s["v_scale"])
        s["decay"] = [DECAY if n > c["width"] else 0.0 for n in sizes]           # none for the vectors
        if own:
            import paper_2003_11666_b200 as pb
            v = s["lists"]
            s["plan"] = pb.AdamW(v["w"], v["m"], v["v"], m_scale=v.get("m_scale"), v_scale=v.get("v_scale"), w_forward=v.get("forward"),
                                 weight_decay=s["decay"], horizon=c["horizon"])
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if own:
        import paper_2003_11666_b200 as pb
        if op == "embed_forward":
            pb.embed_forward(s["table"], s["ids"], s["out"], scale=s["scale"])
            return s["out"]
        if op == "embed_backward":
            pb.embed_backward(s["dout"], s["ids"], s["dtable"], s["scratch"], scale=s["scale"], padding_idx=s["pad"], accumulate=c["accumulate"])
            return s["dtable"]
        if op == "logprob_forward":
            pb.logprob_forward(s["logits"], s["tokens"], s["logp"], entropy=s["entropy"], lse=s["lse"], top_logp=s["top_logp"], top_ids=s["top_ids"],
                               inv_temperature=s["it"])
            return {k: s[k] for k in ("logp", "entropy", "lse", "top_logp", "top_ids")}
        if op == "logprob_backward":
            pb.logprob_backward(s["logits"], s["tokens"], s["lse"], s["dlogits"], g_logp=s["g_logp"], g_entropy=s["g_entropy"], entropy=s["entropy"],
                                inv_temperature=s["it"])
            return s["dlogits"]
        s["step"] += 1
        s["plan"].step(s["lists"]["grad"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, step=s["step"], seed=s["seed"], grad_scale=s["scale"])
        if c["bits"] == 8:
            pb.adamw_moments(s["m"], s["m_scale"], s["v"], s["v_scale"], s["m_read"], s["v_read"])
            return {"w": s["w"], "m": s["m_read"], "v": s["v_read"], "forward": s["forward"]}
        return {k: s[k] for k in ("w", "m", "v", "forward")}
    if op == "embed_forward":
        return _embed_forward(s["table"], s["ids"], s["scale"])
    if op == "embed_backward":
        return _embed_backward(s["dout"], s["ids"], s["dtable"], s["scale"], s["pad"], c["accumulate"])
    if op == "logprob_forward":
        return _logprob_forward(s["logits"], s["tokens"], s["it"], c["top"])
    if op == "logprob_backward":
        return _logprob_backward(s["logits"], s["tokens"], s["lse"], s["entropy"], s["g_logp"], s["g_entropy"], s["it"])
    s["step"] += 1
    for k in range(len(s["sizes"])):
        _adamw(s, k, c)
    if c["bits"] == 8:
        return {"w": s["w"], "m": _read_m(s["m"], s["m_scale"]).reshape(-1), "v": _read_r(s["v"], s["v_scale"]).square().reshape(-1), "forward": s["forward"]}
    return {k: s[k] for k in ("w", "m", "v", "forward")}


def _embed_forward(table, ids, scale):
    there = ids >= 0
    rows = table[ids.long().clamp(min=0)].float() * scale
    return torch.where(there[:, None], rows, 0.0).to(table.dtype)


def _embed_backward(dout, ids, dtable, scale, pad, accumulate):
    # in 64 bits: a frequent token's row is a sum of thousands
    there = (ids >= 0) & (ids != pad)
    total = torch.zeros(dtable.shape, dtype=torch.float64, device=dtable.device)
    total.index_add_(0, ids.long().clamp(min=0), torch.where(there[:, None], dout.double(), 0.0))
    total *= scale
    if accumulate:
        total += dtable
    return dtable.copy_(total)


def _logprob_forward(x, tok, it, k):
    # sums, and the difference of a token's logit and their logarithm, in 64 bits: a confident row's values are near zero
    x = x.float()
    top = x.amax(1, keepdim=True)
    d = (x - top) * it
    e = d.exp()
    z = e.sum(1, keepdim=True, dtype=torch.float64)
    log_z = z.log()
    entropy = log_z - (e * torch.where(e > 0, d, 0.0)).sum(1, keepdim=True, dtype=torch.float64) / z
    logp = (x.gather(1, tok.long().clamp(min=0)[:, None]) - top).double() * it - log_z
    logp = torch.where(tok[:, None] >= 0, logp, 0.0)
    del d, e
    # top alternatives: 64-bit keys, the logit's order in the upper half, the lower index first among equal ones
    bits = (x + 0.0).view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + ((1 << 32) - 1 - torch.arange(x.shape[1], device=x.device))
    ids = (1 << 32) - 1 - (key.topk(k, 1).values & 0xFFFFFFFF)
    top_logp = (x.gather(1, ids) - top).double() * it - log_z
    ids = torch.where(top_logp > -math.inf, ids, -1)
    f = lambda v: v.float()                                                      # noqa: E731
    return {"logp": f(logp[:, 0]), "entropy": f(entropy[:, 0]), "lse": f((top.double() * it + log_z)[:, 0]), "top_logp": f(top_logp),
            "top_ids": ids.to(torch.int32)}


def _logprob_backward(x, tok, lse, entropy, g_logp, g_entropy, it):
    lp = (x.double() * it - lse[:, None]).float()
    p = lp.exp()
    there = (tok >= 0)[:, None]
    at = tok.long().clamp(min=0)[:, None]
    gl = torch.where(there, g_logp[:, None], 0.0)
    h = g_entropy[:, None] * p * (torch.where(p > 0, lp, 0.0) + entropy[:, None])
    # the given token: 1 - p without the cancellation
    d = (-gl * p).scatter(1, at, torch.where(there, -gl * torch.expm1(lp.gather(1, at)), 0.0))
    return ((d - h) * it).to(x.dtype)


def _read_m(code, scale):
    return code.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * scale[:, None]


def _read_r(code, scale):
    code = code.to(torch.int32)
    r = torch.where(code > 0, ((code + 1792) << 19).view(torch.float32), 0.0)
    return r.view(-1, BLOCK) * scale[:, None]


def _signed(c):
    return c - (1 << 64) if c >= 1 << 63 else c


def _random16(seed, stream, n, device):
    """16 random bits for each of n elements (n a multiple of 4): SplitMix64 of a counter for four elements."""
    base = (seed * 0xD1342543DE82EF95 + stream * 0xA0761D6478BD642F) % (1 << 64)
    z = (torch.arange(n // 4, device=device) + 1) * _signed(0x9E3779B97F4A7C15) + _signed(base)
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    z = z ^ ((z >> 31) & ((1 << 33) - 1))
    return ((z[:, None] >> torch.tensor([0, 16, 32, 48], device=device)) & 0xFFFF).to(torch.int32).reshape(-1)


def _adamw(s, k, c):
    v = s["lists"]
    w, n, t = v["w"][k], s["sizes"][k], s["step"]
    g = v["grad"][k].float() * s["scale"]
    if c["bits"] == 8:
        full = -(-n // BLOCK) * BLOCK
        m_codes, v_codes = torch.zeros(full, dtype=torch.uint8, device=w.device), torch.zeros(full, dtype=torch.uint8, device=w.device)
        m_codes[:n], v_codes[:n] = v["m"][k], v["v"][k]
        m = _read_m(m_codes, v["m_scale"][k]).reshape(-1)[:n]
        q = _read_r(v_codes, v["v_scale"][k]).square().reshape(-1)[:n]
    else:
        m, q = v["m"][k], v["v"][k]
    # each operation rounded to float32, as the moments are defined: the codes of an 8-bit state follow from them
    m = m * BETA1 + g * (1 - BETA1)
    q = q * BETA2 + (g * (1 - BETA2)) * g
    r = q.sqrt()
    u = (m * (1 / (1 - BETA1 ** t))) / (r * (1 / math.sqrt(1 - BETA2 ** t)) + EPS)
    w.copy_(w * (1 - LR * s["decay"][k]) - u * LR)
    if s["forward"] is not None:
        v["forward"][k].copy_(w - u * (LR * c["horizon"]))
    if c["bits"] == 32:
        v["m"][k].copy_(m)
        v["v"][k].copy_(q)
        return
    pad = lambda x: torch.cat([x, x.new_zeros(full - n)]).view(-1, BLOCK)        # noqa: E731
    mb, rb = pad(m), pad(r)
    ma, ra = mb.abs().amax(1, keepdim=True), rb.amax(1, keepdim=True)
    live = ma >= 2.0 ** -100
    x = torch.where(live, mb * (torch.full_like(ma, 448.0) / ma), 0.0)
    v["m"][k].copy_(x.to(torch.float8_e4m3fn).view(torch.uint8).reshape(-1)[:n])
    v["m_scale"][k].copy_(torch.where(live, ma / 448.0, 0.0).reshape(-1))
    x = rb * torch.where(ra > 0, torch.full_like(ra, 1.9375) / ra, 0.0)
    noise = _random16(s["seed"] + t, k, full, w.device).view(-1, BLOCK) << 3
    code = ((x.view(torch.int32) + noise) >> 19) - 1792
    v["v"][k].copy_(torch.where(rb > 0, code.clamp(1, 255), 0).to(torch.uint8).reshape(-1)[:n])
    v["v_scale"][k].copy_((ra / torch.full_like(ra, 1.9375)).reshape(-1))


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c, op = case, case["op"]
    f = torch.float64
    if op == "embed_forward":
        out = torch.zeros(c["tokens"], c["dim"], dtype=f, device=DEV)
        live = (s["ids"] >= 0).nonzero()[:, 0]
        out[live] = s["table"].index_select(0, s["ids"][live].long()).to(f) * s["scale"]
        return out
    if op == "embed_backward":
        order = torch.argsort(s["ids"], stable=True)
        ids = s["ids"][order].long()
        keep = (ids >= 0) & (ids != s["pad"])
        order, ids = order[keep], ids[keep]
        total = s["dtable"].to(f) if c["accumulate"] else torch.zeros(c["vocab"], c["dim"], dtype=f, device=DEV)
        if ids.numel() and c["dim"]:
            rows, counts = torch.unique_consecutive(ids, return_counts=True)
            run_sums = torch.cat([torch.zeros(1, c["dim"], dtype=f, device=DEV), s["dout"][order].to(f).cumsum(0)])
            ends = counts.cumsum(0)
            total[rows] += (run_sums[ends] - run_sums[ends - counts]) * s["scale"]
        return total
    if op == "logprob_forward":
        got = [[], [], [], []]
        for x, tok in zip(s["logits"].split(max(1, (1 << 27) // c["vocab"])), s["tokens"].split(max(1, (1 << 27) // c["vocab"]))):
            lp = torch.log_softmax(x.to(f) * s["it"], 1)
            got[0].append(torch.where(tok >= 0, lp[torch.arange(len(tok), device=DEV), tok.long().clamp(min=0)], 0.0))
            got[1].append(torch.special.entr(lp.exp()).sum(1))
            got[2].append(torch.logsumexp(x.to(f) * s["it"], 1))
            got[3].append(lp.topk(c["top"], 1).values)
        logp, entropy, lse, top = (torch.cat(v) for v in got)
        return {"logp": logp, "entropy": entropy, "lse": lse, "top_logp": top, "top_ids": None}
    if op == "logprob_backward":
        got = []
        for k in range(0, c["rows"], max(1, (1 << 26) // c["vocab"])):
            at = slice(k, k + max(1, (1 << 26) // c["vocab"]))
            x, tok = s["logits"][at].to(f), s["tokens"][at].long()
            lp = x * s["it"] - s["lse"][at, None].to(f)
            gl = s["g_logp"][at].to(f) * (tok >= 0)
            hot = torch.arange(c["vocab"], device=DEV)[None] == tok[:, None]
            d = gl[:, None] * (hot.to(f) - lp.exp()) + s["g_entropy"][at, None].to(f) * (torch.special.entr(lp.exp()) - lp.exp() * s["entropy"][at, None].to(f))
            got.append((d * s["it"]).float())       # gradients: 32 bits hold them to 6e-8
        return torch.cat(got)
    t = s["step"] + 1
    both = {"w": [], "m": [], "v": [], "forward": []}
    g = s["grad"].to(f) * s["scale"].to(f)
    if c["bits"] == 8:
        m = s["m"].view(torch.float8_e4m3fn).to(f) * s["m_scale"].to(f).repeat_interleave(BLOCK)
        code = s["v"].to(f)
        r = torch.where(code > 0, torch.exp2(torch.floor(code / 16) - 15) * (1 + torch.remainder(code, 16) / 16), 0.0) * s["v_scale"].to(f).repeat_interleave(BLOCK)
        q = r * r
    else:
        m, q = s["m"].to(f), s["v"].to(f)
    m, q = m + (1 - BETA1) * (g - m), q + (1 - BETA2) * (g * g - q)
    w, forward = s["w"].to(f), None if s["forward"] is None else s["forward"].to(f)
    new_w, new_m, new_q = w.clone(), s["m"].clone(), s["v"].clone()
    if c["bits"] == 32:
        new_m, new_q = new_m.to(f), new_q.to(f)
    for k, n in enumerate(s["sizes"]):
        a = s["lists"]["w"][k].storage_offset()
        at = slice(a, a + n)
        u = m[at] / (1 - BETA1 ** t) / ((q[at] / (1 - BETA2 ** t)).sqrt() + EPS)
        new_w[at] = w[at] - LR * s["decay"][k] * w[at] - LR * u
        if forward is not None:
            forward[at] = new_w[at] - LR * c["horizon"] * u
        if c["bits"] == 32:
            new_m[at], new_q[at] = m[at], q[at]
    # what is rounded to 8 bits (the second moment at random) has no 64-bit value
    return {"w": new_w, "m": new_m if c["bits"] == 32 else None, "v": new_q if c["bits"] == 32 else None, "forward": forward}
