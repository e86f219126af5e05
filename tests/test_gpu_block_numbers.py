"""Numbers that are none, or that the C argument cannot hold: PBError with code -1, as for tensors that do not fit."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_numbers_that_do_not_fit_are_refused():
    import paper_2003_11666_b200 as p
    f = lambda *n: torch.zeros(*n, device="cuda")                 # noqa: E731
    h, w, tok = f(4, 8), f(10, 8), torch.zeros(4, dtype=torch.int64, device="cuda")
    byte = lambda n: torch.zeros(n, device="cuda", dtype=torch.uint8)              # noqa: E731
    sf, sb, sj = byte(p.head_scratch_bytes(h, w)), byte(p.head_scratch_bytes(h, w, True)), byte(p.join_scratch_bytes(4, 8))
    fwd = lambda **k: p.join_forward(h, f(4, 8), f(4, 8), **k)     # noqa: E731
    back = lambda **k: p.join_backward(h, f(4, 8), f(4, 8), f(4, 8), sj, dy=f(4, 8), **k)      # noqa: E731
    calls = [lambda k=k, v=v, c=c: c(**{k: v}) for c in (fwd, back) for k, v in (("residual_scale", 1e60), ("residual_scale", "a"), ("p", None), ("p", 10 ** 400), ("seed", 1.5),
                                                                                 ("offset", 1 << 63), ("offset", 0.5), ("stream", 1.5))]
    calls += [lambda: fwd(eps=1e60), lambda: fwd(gate=f(1, 8), rows_per_gate="a"), lambda: fwd(gate=f(1, 8), rows_per_gate=1 << 63)]
    calls += [lambda k=k: p.dropout(h, f(4, 8), **{**dict(p=0.5, seed=1), **k}) for k in (dict(p=10 ** 400), dict(seed=None), dict(offset=0.5), dict(stream=0.5), dict(offset=1 << 63),
                                                                                         dict(offset=-(1 << 63) - 1))]
    for bad in ("a", None, 10 ** 400, f(2)):
        calls += [lambda b=bad: p.head_logprob_forward(h, w, sf, tok, f(4), inv_temperature=b), lambda b=bad: p.head_logprob_backward(h, w, sb, tok, f(4), f(4, 8), inv_temperature=b)]
    calls += [lambda: p.head_logprob_forward(h, w, sf, tok, f(4), stream=0.5), lambda: p.head_logprob_backward(h, w, sb, tok, f(4), f(4, 8), stream=0.5)]
    for k, call in enumerate(calls):
        with pytest.raises(p.PBError) as e:
            call()
        assert e.value.code == -1, k
