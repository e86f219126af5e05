"""AdamW over tensors whose memory is replaced between steps."""
import pytest

pytestmark = pytest.mark.gpu


def _make(torch, bits):
    g = torch.Generator(device="cuda")
    g.manual_seed(bits)
    sizes = [700, 256, 33]
    rand = lambda n: torch.randn(n, generator=g, device="cuda")    # noqa: E731
    w, grads = [torch.nn.Parameter(rand(n)) for n in sizes], [rand(n) for n in sizes]
    kind = torch.uint8 if bits == 8 else torch.float32
    m, v = ([torch.zeros(n, device="cuda", dtype=kind) for n in sizes] for _ in range(2))
    scales = [[torch.zeros(-(-n // 256), device="cuda") for n in sizes] for _ in range(2)] if bits == 8 else [None, None]
    return w, grads, m, v, scales, [torch.zeros(n, device="cuda", dtype=torch.bfloat16) for n in sizes]


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_follow_tensors_that_moved(bits):
    import torch
    import paper_2003_11666_b200 as p
    both = [_make(torch, bits) for _ in range(2)]
    plans = [p.AdamW(w, m, v, m_scale=s[0], v_scale=s[1], w_forward=f, weight_decay=0.1) for w, _, m, v, s, f in both]
    held = []
    for step in (1, 2, 3, 4):
        w, grads, m, v, scales, f = both[1]
        old = None
        if step in (2, 3):                                         # the weights, then their copies
            for t in (w, f)[step - 2]:
                old = t.data
                t.data = t.data.clone()
            before = old.clone()
        if step == 4:                                              # the states are the object's: other tensors' memory is not
            for t in m + v:
                held.append(t.data)
                t.data = torch.ones_like(t)
        for (_, g, *_), plan in zip(both, plans):
            plan.step(g, lr=0.01, step=step, seed=3)
        if old is not None:
            assert torch.equal(old, before)                        # memory that was given up is not written
        for t, was in zip(m + v, held):
            assert (t == 1).all()
            t.data = was
        for x, y in zip(both[0], both[1]):
            for a, b in zip(x, y):
                for q, r in zip(a, b) if isinstance(a, list) else [(a, b)]:
                    if q is not None:
                        assert torch.equal(q, r)


def test_tensors_that_no_longer_fit_are_refused():
    import torch
    import paper_2003_11666_b200 as p
    w, grads, m, v, _, _ = _make(torch, 32)
    plan = p.AdamW(w, m, v)
    plan.step(grads, lr=0.01, step=1)
    good = w[1].data
    for bad in (good[:100].clone(), good.double(), good.cpu(), m[1].data):
        w[1].data = bad
        for _ in range(2):                                         # and go on being refused
            with pytest.raises(p.PBError) as e:
                plan.step(grads, lr=0.01, step=2)
            assert e.value.code == -1
    w[1].data = good
    plan.step(grads, lr=0.01, step=2)
    assert torch.isfinite(w[1]).all()
