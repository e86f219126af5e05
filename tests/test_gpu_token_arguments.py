"""Arguments of the token operators that are no tensors, or are missing: PBError with code -1, like all that does not
fit."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_what_is_no_tensor_is_refused():
    import torch
    import paper_2003_11666_b200 as p
    f = lambda *n: torch.zeros(*n, device="cuda")                 # noqa: E731
    u8 = lambda n: torch.zeros(n, device="cuda", dtype=torch.uint8)          # noqa: E731
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    scratch = u8(p.embed_scratch_bytes(4, 10, 8))
    plan = p.AdamW([f(5), f(6)], [f(5), f(6)], [f(5), f(6)])
    host, numbers = np.zeros(4, np.int64), [0, 1, 2, 3]
    calls = []
    for bad in (None, host, numbers):
        calls += [lambda b=bad: p.embed_forward(f(10, 8), b, f(4, 8)), lambda b=bad: p.embed_forward(f(10, 8), ids, b),
                  lambda b=bad: p.embed_forward(b, ids, f(4, 8)), lambda b=bad: p.embed_backward(b, ids, f(10, 8), scratch),
                  lambda b=bad: p.embed_backward(f(4, 8), b, f(10, 8), scratch), lambda b=bad: p.embed_backward(f(4, 8), ids, b, scratch),
                  lambda b=bad: p.embed_backward(f(4, 8), ids, f(10, 8), b), lambda b=bad: p.logprob_forward(b, ids, f(4)),
                  lambda b=bad: p.logprob_forward(f(4, 8), ids, b), lambda b=bad: p.logprob_backward(b, ids, f(4), f(4, 8)),
                  lambda b=bad: p.logprob_backward(f(4, 8), ids, b, f(4, 8)), lambda b=bad: p.logprob_backward(f(4, 8), ids, f(4), b),
                  lambda b=bad: p.adamw_moments(b, f(1), u8(5), f(1), f(5), f(5)), lambda b=bad: p.adamw_moments(u8(5), b, u8(5), f(1), f(5), f(5)),
                  lambda b=bad: p.AdamW([b], [f(5)], [f(5)]), lambda b=bad: p.AdamW([f(5)], [b], [f(5)]), lambda b=bad: p.AdamW([f(5)], [f(5)], [b]),
                  lambda b=bad: plan.step([f(5), b], lr=0.1, step=1), lambda b=bad: plan.step([b, f(6)], lr=0.1, step=1)]
        if bad is not None:
            calls += [lambda b=bad: p.logprob_forward(f(4, 8), b, f(4)), lambda b=bad: p.logprob_forward(f(4, 8), ids, f(4), status=b),
                      lambda b=bad: p.logprob_forward(f(4, 8), ids, f(4), top_logp=b, top_ids=b), lambda b=bad: p.AdamW([f(5)], [f(5)], [f(5)], w_forward=[b]),
                      lambda b=bad: p.AdamW([f(5)], [u8(5)], [u8(5)], m_scale=[b], v_scale=[f(1)]),
                      lambda b=bad: plan.step([f(5), f(6)], lr=0.1, step=1, grad_scale=b)]
    for call in calls:
        with pytest.raises(p.PBError) as e:
            call()
        assert e.value.code == -1
