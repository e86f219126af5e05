"""A token operator reports its own launch, not an error that an earlier call of the library has left and reported."""
import pytest

pytestmark = pytest.mark.gpu


def test_an_earlier_failed_create_is_not_reported_again():
    import torch
    import paper_2003_11666_b200 as p
    from pb_workloads import mlp
    f = lambda *n: torch.ones(*n, device="cuda")                  # noqa: E731
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    scratch = torch.empty(p.embed_scratch_bytes(4, 10, 8), dtype=torch.uint8, device="cuda")
    big = torch.empty(p.embed_scratch_bytes(5000, 10, 8), dtype=torch.uint8, device="cuda")
    many = torch.zeros(5000, dtype=torch.int64, device="cuda")
    plan = p.AdamW([f(5)], [f(5)], [f(5)])
    u8 = torch.zeros(5, dtype=torch.uint8, device="cuda")
    calls = [lambda: p.embed_forward(f(10, 8), ids, f(4, 8)), lambda: p.embed_backward(f(4, 8), ids, f(10, 8), scratch),
             lambda: p.embed_backward(f(5000, 8), many, f(10, 8), big), lambda: p.logprob_forward(f(4, 8), ids, f(4)),
             lambda: p.logprob_forward(f(1, 100000), None, None, lse=f(1)), lambda: p.logprob_backward(f(4, 8), ids, f(4), f(4, 8)),
             lambda: plan.step([f(5)], lr=0.1, step=1), lambda: p.adamw_moments(u8, f(1), u8, f(1), f(5), f(5))]
    wl = mlp([400_000, 400_000, 10], lr=0.01, seed=1)              # weights and velocity: 1.3 TB, more than any device has
    for call in calls:
        with pytest.raises(p.PBError, match="cudaMalloc"):
            p.PB(wl.layers, wl.stage_of_layer, wl.in_shape, wl.n_classes, wl.lr, wl.momentum, wl.flags)
        call()
    torch.cuda.synchronize()
