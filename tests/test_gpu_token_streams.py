"""The token operators on torch's streams: without an argument they run on the current one."""
import pytest

pytestmark = pytest.mark.gpu


def _state(torch, p):
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    e = lambda *n, d=torch.float32: torch.zeros(*n, device="cuda", dtype=d)    # noqa: E731
    vocab, dim, n = 3000, 64, 500
    s = dict(src=rand(vocab, dim), table=e(vocab, dim), ids=torch.randint(0, vocab, (n,), generator=g, device="cuda"), x=e(n, dim),
             logits_src=rand(n, vocab), logits=e(n, vocab), logp=e(n), lse=e(n), ent=e(n), top=e(n, 3), tid=e(n, 3, d=torch.int32), dlogits=e(n, vocab),
             dtable=e(vocab, dim), scratch=e(p.embed_scratch_bytes(n, vocab, dim), d=torch.uint8), gl=e(n) - 1.0)
    size = vocab * dim
    s.update(w=rand(vocab, dim), m=e(size, d=torch.uint8), v=e(size, d=torch.uint8), ms=e(-(-size // 256)), vs=e(-(-size // 256)), mo=e(size), vo=e(size))
    s["plan"] = p.AdamW([s["w"]], [s["m"]], [s["v"]], m_scale=[s["ms"]], v_scale=[s["vs"]])
    return s


def _step(p, s):
    """Every function once, each on what torch or the one before has made on the same stream."""
    s["table"].copy_(s["src"])
    p.embed_forward(s["table"], s["ids"], s["x"])
    s["logits"].copy_(s["logits_src"])
    p.logprob_forward(s["logits"], s["ids"], s["logp"], entropy=s["ent"], lse=s["lse"], top_logp=s["top"], top_ids=s["tid"])
    p.logprob_backward(s["logits"], s["ids"], s["lse"], s["dlogits"], g_logp=s["gl"])
    p.embed_backward(s["x"], s["ids"], s["dtable"], s["scratch"])
    s["plan"].step([s["dtable"]], lr=0.01, step=1)
    p.adamw_moments(s["m"], s["ms"], s["v"], s["vs"], s["mo"], s["vo"])


RESULTS = ("x", "logp", "lse", "ent", "top", "tid", "dlogits", "dtable", "w", "m", "v", "ms", "vs", "mo", "vo")


def _same(torch, a, b):
    for k in RESULTS:
        assert torch.equal(a[k], b[k]), k


def test_calls_follow_the_current_stream():
    import torch
    import paper_2003_11666_b200 as p
    ref, got = _state(torch, p), _state(torch, p)
    _step(p, ref)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(50_000_000)                              # what runs elsewhere comes too early
        _step(p, got)
    stream.synchronize()
    torch.cuda.synchronize()
    _same(torch, ref, got)


def test_calls_are_captured_on_the_capturing_stream():
    import torch
    import paper_2003_11666_b200 as p
    ref, got = _state(torch, p), _state(torch, p)
    _step(p, ref)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(p, got)
    assert not got["x"].any() and not got["logp"].any()            # nothing has run yet
    graph.replay()
    torch.cuda.synchronize()
    _same(torch, ref, got)


def test_an_integer_names_another_stream():
    import torch
    import paper_2003_11666_b200 as p
    s, stream = _state(torch, p), torch.cuda.Stream()
    s["table"].copy_(s["src"])
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(50_000_000)
        p.embed_forward(s["table"], s["ids"], s["x"], stream=0)
        torch.cuda.default_stream().synchronize()
        assert torch.equal(s["x"].cpu(), s["src"].cpu()[s["ids"].cpu()])
