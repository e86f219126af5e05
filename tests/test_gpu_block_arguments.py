"""Arguments of the head, join and dropout operators that are no tensors, are missing or do not fit: PBError with code -1."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_what_does_not_fit_is_refused():
    import torch
    import paper_2003_11666_b200 as p
    f = lambda *n: torch.zeros(*n, device="cuda")                 # noqa: E731
    u8 = lambda n: torch.zeros(n, device="cuda", dtype=torch.uint8)          # noqa: E731
    h, w, tok = f(4, 8), f(10, 8), torch.zeros(4, dtype=torch.int64, device="cuda")
    sf, sb, sj = u8(p.head_scratch_bytes(h, w)), u8(p.head_scratch_bytes(h, w, True)), u8(p.join_scratch_bytes(4, 8, 1))
    back = lambda **k: p.join_backward(**{**dict(y=f(4, 8), u=f(4, 8), dx=f(4, 8), du=f(4, 8), scratch=sj, dy=f(4, 8)), **k})      # noqa: E731
    fwd = lambda **k: p.join_forward(**{**dict(x=f(4, 8), u=f(4, 8), y=f(4, 8)), **k})                                            # noqa: E731
    calls = []
    for bad in (np.zeros((4, 8)), [1, 2], f(4, 9), f(5, 8), f(4, 8).cpu(), f(8, 4).t(), f(4, 8).to(torch.int32)):
        calls += [lambda b=bad: p.head_logprob_forward(b, w, sf, tok, f(4)),
                  lambda b=bad: p.head_logprob_backward(h, w, sb, tok, f(4), dhidden=b, g_logp=f(4)), lambda b=bad: p.head_logprob_forward(h, w, sf, b, f(4)),
                  lambda b=bad: p.head_logprob_forward(h, w, b, tok, f(4)), lambda b=bad: p.head_logprob_backward(h, w, sb, tok, b, dhidden=f(4, 8)),
                  lambda b=bad: p.head_logprob_backward(h, w, sb, tok, f(4), dweight=b), lambda b=bad: p.head_logprob_forward(h, w, sf, tok, f(4), status=b)]
        calls += [lambda b=bad, n=n: fwd(**{n: b}) for n in ("x", "u", "y", "h", "pre_weight", "post_weight", "rstd_pre", "dev_offset")]
        calls += [lambda b=bad, n=n: back(**{n: b}) for n in ("y", "dx", "du", "dy", "dh", "scratch", "post_weight", "dpost_weight", "rstd_post", "dgate")]
        calls += [lambda b=bad: p.dropout(b, f(4, 8), 0.5, 1) if not torch.is_tensor(b) or b.shape != (4, 8) else p.dropout(b, f(3, 8), 0.5, 1),
                  lambda b=bad: p.dropout(f(4, 8), b, 0.5, 1), lambda b=bad: p.dropout(f(4, 8), f(4, 8), 0.5, 1, dev_offset=b)]
    calls += [lambda: p.head_logprob_forward(h, w, sf, tok), lambda: p.head_logprob_forward(h, w, sf, None, f(4)), lambda: p.head_logprob_forward(h, w.half(), sf),
              lambda: p.head_logprob_forward(h, w, u8(1)), lambda: p.head_logprob_forward(h, w, None), lambda: p.head_logprob_backward(h, w, sb, tok, None, f(4, 8)),
              lambda: p.head_logprob_backward(h, w, sb, tok, f(4)), lambda: p.head_logprob_backward(h, w, sb, None, f(4), f(4, 8), g_logp=f(4)),
              lambda: p.head_logprob_backward(h, w, sf[:1], tok, f(4), f(4, 8)), lambda: fwd(gate=f(1, 8), rows_per_gate=2), lambda: fwd(gate=f(4, 8), rows_per_gate=0),
              lambda: fwd(gate=f(4, 8), rows_per_gate=-1), lambda: fwd(pre_weight=f(8)), lambda: fwd(h=f(4, 8)), lambda: fwd(p=1.0), lambda: fwd(eps="a"),
              lambda: fwd(pre_weight=f(8).half(), post_weight=f(8), h=f(4, 8)), lambda: back(dgate=f(1, 8)), lambda: back(dy=None), lambda: back(dh=f(4, 8)),
              lambda: back(dpre_weight=f(8)), lambda: back(scratch=None), lambda: back(du=None), lambda: p.dropout(h, h, 1.0, 1), lambda: p.dropout(h, h, "a", 1),
              lambda: p.dropout(h, None, 0.5, 1), lambda: p.dropout(f(8), f(8), 0.5, 1), lambda: p.join_forward(None, h, h), lambda: p.join_forward(h, None, h)]
    for k, call in enumerate(calls):
        with pytest.raises(p.PBError) as e:
            call()
        assert e.value.code == -1, k


def test_views_of_one_row_and_one_column_are_taken_as_they_lie():
    import torch
    import paper_2003_11666_b200 as p
    big = torch.randn(40, 30, device="cuda")
    row, column = big[3:4, :8], big[:, 5:6]
    out = torch.empty(1, 8, device="cuda")
    p.dropout(row, out, 0.0, 1)
    assert torch.equal(out, row)
    out = torch.empty(40, 1, device="cuda")
    p.dropout(column, out, 0.0, 1)
    assert torch.equal(out, column)
    y = torch.empty(40, 1, device="cuda")
    p.join_forward(column, column, y, residual_scale=2.0)
    assert torch.equal(y, 3.0 * column)
    lse = torch.empty(1, device="cuda")
    w = torch.randn(50, 8, device="cuda")
    p.head_logprob_forward(row, w, torch.empty(p.head_scratch_bytes(row, w), device="cuda", dtype=torch.uint8), lse=lse)
    assert abs(float(lse) - float((row.double() @ w.double().T).logsumexp(1))) < 2.0 ** -18
