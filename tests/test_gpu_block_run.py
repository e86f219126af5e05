"""A training step of a small model through all token operators: embedding, dropout, two blocks joined to the residual
stream, log probabilities under the tied head, every gradient, AdamW.  And the scoring of single tokens."""
import pytest
import torch

from tests import blocks_ref as R

pytestmark = pytest.mark.gpu

VOCAB, DIM, ROWS, P, EPS = 1000, 64, 150, 0.2, 1e-5
WEIGHTS = [("table", (VOCAB, DIM)), ("w0", (DIM, DIM)), ("w1", (DIM, DIM)), ("post0", (DIM,)), ("post1", (DIM,)), ("pre0", (DIM,)), ("pre1", (DIM,)),
           ("gate0", (1, DIM)), ("gate1", (1, DIM))]


def _model(seed):
    import paper_2003_11666_b200 as p
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    z = lambda *n, d=torch.float32: torch.zeros(*n, device="cuda", dtype=d)      # noqa: E731
    s = {n: rand(*shape) * 0.1 if len(shape) == 2 else rand(*shape).abs() + 0.5 for n, shape in WEIGHTS}
    s["gate0"] += 1.0
    s["ids"] = torch.randint(0, VOCAB, (ROWS,), generator=g, device="cuda")
    s["ids"][7] = -1
    s["next"] = torch.randint(0, VOCAB, (ROWS,), generator=g, device="cuda")
    s["next"][11] = -1
    for n in ("e", "x0", "x1", "x2", "h0", "h1", "u0", "u1", "dx", "dh0", "dh1", "du0", "du1", "tmp"):
        s[n] = z(ROWS, DIM)
    for n in ("logp", "lse", "ent", "rp0", "rp1", "rr0", "rr1"):
        s[n] = z(ROWS)
    s["gl"], s["ge"] = torch.full((ROWS,), -1.0 / ROWS, device="cuda"), torch.full((ROWS,), -0.01 / ROWS, device="cuda")
    s["grads"] = {n: z(*shape) for n, shape in WEIGHTS}
    s["step"] = torch.ones(1, dtype=torch.int64, device="cuda")
    byte = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")          # noqa: E731
    s["hs"], s["hb"] = byte(p.head_scratch_bytes(s["h1"], s["table"])), byte(p.head_scratch_bytes(s["h1"], s["table"], backward=True))
    s["js"], s["es"] = byte(p.join_scratch_bytes(ROWS, DIM, ROWS)), byte(p.embed_scratch_bytes(ROWS, VOCAB, DIM))
    w = [s[n] for n, _ in WEIGHTS]
    s["plan"] = p.AdamW(w, [torch.zeros_like(t) for t in w], [torch.zeros_like(t) for t in w])
    return s


def _gradients(s):
    import paper_2003_11666_b200 as p
    g = s["grads"]
    drop = dict(p=P, seed=5, dev_offset=s["step"])
    join = lambda k: dict(pre_weight=s["pre%d" % k], post_weight=s["post%d" % k], gate=s["gate%d" % k], rstd_pre=s["rr%d" % k],   # noqa: E731
                          rstd_post=s["rp%d" % k], residual_scale=0.9, p=P, seed=6 + k, dev_offset=s["step"])
    p.embed_forward(s["table"], s["ids"], s["e"], scale=3.0)
    p.dropout(s["e"], s["x0"], **drop)
    torch.mm(s["x0"], s["w0"], out=s["u0"])
    p.join_forward(s["x0"], s["u0"], s["x1"], h=s["h0"], eps=EPS, **join(0))
    torch.mm(s["h0"], s["w1"], out=s["u1"])
    p.join_forward(s["x1"], s["u1"], s["x2"], h=s["h1"], eps=EPS, **join(1))
    p.head_logprob_forward(s["h1"], s["table"], s["hs"], s["next"], s["logp"], entropy=s["ent"], lse=s["lse"])
    p.head_logprob_backward(s["h1"], s["table"], s["hb"], s["next"], s["lse"], s["dh1"], g["table"], g_logp=s["gl"], g_entropy=s["ge"], entropy=s["ent"])
    p.join_backward(s["x2"], s["u1"], s["dx"], s["du1"], s["js"], dh=s["dh1"], dgate=g["gate1"], dpost_weight=g["post1"], dpre_weight=g["pre1"], **join(1))
    torch.mm(s["h0"].T, s["du1"], out=g["w1"])
    torch.mm(s["du1"], s["w1"].T, out=s["dh0"])
    p.join_backward(s["x1"], s["u0"], s["dx"], s["du0"], s["js"], dy=s["dx"], dh=s["dh0"], dgate=g["gate0"], dpost_weight=g["post0"], dpre_weight=g["pre0"],
                    **join(0))
    torch.mm(s["x0"].T, s["du0"], out=g["w0"])
    torch.addmm(s["dx"], s["du0"], s["w0"].T, out=s["tmp"])
    p.dropout(s["tmp"], s["dx"], **drop)
    p.embed_backward(s["dx"], s["ids"], g["table"], s["es"], scale=3.0, accumulate=True)


def _step(s):
    _gradients(s)
    s["plan"].step([s["grads"][n] for n, _ in WEIGHTS], lr=1e-3, step=1, dev_step=s["step"])


def _plain(s):
    """Loss and gradients in float64 by autograd."""
    leaf = {n: s[n].double().requires_grad_(True) for n, _ in WEIGHTS}
    k = int(s["step"])
    keep = lambda seed: R.keep(seed, k, P, ROWS, DIM).cuda()        # noqa: E731
    e = torch.where((s["ids"] >= 0)[:, None], 3.0 * leaf["table"][s["ids"].clamp(min=0)], 0.0)
    x = x0 = e * keep(5)
    h = x0
    for b in range(2):
        x, h, _, _ = R.join_forward(x, h @ leaf["w%d" % b], leaf["gate%d" % b], ROWS, leaf["post%d" % b], leaf["pre%d" % b], 0.9, EPS, keep(6 + b))
    lp = torch.log_softmax(h @ leaf["table"].T, 1)
    at = torch.where(s["next"] >= 0, lp[torch.arange(ROWS), s["next"].clamp(min=0)], 0.0)
    ent = -(lp.exp() * lp).sum(1)
    (-at.sum() / ROWS - 0.01 / ROWS * ent.sum()).backward()
    return at, ent, {n: t.grad for n, t in leaf.items()}


def test_a_training_step_of_all_of_them():
    s = _model(1)
    _gradients(s)
    at, ent, grads = _plain(s)
    # float32 throughout (torch's products too): chains of some ten operations, each good to a few 2^-24 of the root of its
    # terms' squares, sums of 150 rows and 1000 tokens
    for got, ref in [(s["logp"], at), (s["ent"], ent)] + [(s["grads"][n], grads[n]) for n, _ in WEIGHTS]:
        assert float((got.double() - ref).norm() / ref.norm()) < 200 * 2.0 ** -24


def test_captured_steps_replay_and_do_not_share():
    eager, captured = [_model(k) for k in (1, 2)], [_model(k) for k in (1, 2)]
    streams, graphs = [torch.cuda.Stream() for _ in range(2)], []
    for s, stream in zip(captured, streams):
        warm = _model(9)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            _step(warm)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            _step(s)
            s["step"].add_(1)
        graphs.append(graph)
    for _ in range(3):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for s in eager:
            _step(s)
            s["step"].add_(1)
        torch.cuda.synchronize()
    for a, b in zip(eager, captured):
        assert int(a["step"]) == 4
        for n, _ in WEIGHTS:
            assert torch.equal(a[n], b[n]), n


def test_single_tokens_are_scored_as_a_batch_is():
    import paper_2003_11666_b200 as p
    s = _model(3)
    _gradients(s)
    batch, w = s["logp"].clone(), s["table"]
    one, lse = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    for r in (0, 11, 149):
        y, h = torch.empty(1, DIM, device="cuda"), torch.empty(1, DIM, device="cuda")
        # the last join of this token alone, without dropout here, then its score
        p.join_forward(s["x1"][r:r + 1], s["u1"][r:r + 1], y, h=h, pre_weight=s["pre1"], post_weight=s["post1"], gate=s["gate1"], residual_scale=0.9, eps=EPS)
        z, hr, _, _ = R.join_forward(s["x1"][r:r + 1], s["u1"][r:r + 1], s["gate1"], 1, s["post1"], s["pre1"], 0.9, EPS, None)
        p.head_logprob_forward(h, w, s["hs"], s["next"][r:r + 1], one, lse=lse)
        ref, _, _, _ = R.head_forward(hr, w, s["next"][r:r + 1], 1.0)
        assert abs(float(one) - float(ref)) < 2.0 ** -18
        p.head_logprob_forward(s["h1"][r:r + 1], w, s["hs"], s["next"][r:r + 1], one)
        assert abs(float(one) - float(batch[r])) <= 2.0 ** -19
