"""A scratch laid out for a program's largest batch serves its shorter ones."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("most,dim,per", [(7200, 40, 1000), (1400, 1024, 700), (2000, 4096, 300), (7200, 24, 7200)])
def test_shorter_batches_in_the_scratch_of_the_longest(most, dim, per):
    import paper_2003_11666_b200 as p
    g = torch.Generator(device="cuda").manual_seed(dim)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    y, u, dy, dh, w, gates = rand(most, dim), rand(most, dim), rand(most, dim), rand(most, dim), rand(dim), rand(-(-most // per), dim)
    rr, rp = rand(most).abs(), rand(most).abs()
    byte = lambda n: torch.empty(p.join_scratch_bytes(n, dim, per), device="cuda", dtype=torch.uint8)          # noqa: E731
    scratch = byte(most)

    def step(n, s):
        gate = gates[:-(-n // per)]
        out = [torch.empty(n, dim, device="cuda") for _ in range(2)] + [torch.empty(dim, device="cuda") for _ in range(2)] + [torch.empty_like(gate)]
        p.join_backward(y[:n], u[:n], out[0], out[1], s, dy=dy[:n], dh=dh[:n], pre_weight=w, post_weight=w, gate=gate, rows_per_gate=per, rstd_pre=rr[:n], rstd_post=rp[:n],
                        dpre_weight=out[2], dpost_weight=out[3], dgate=out[4])
        return out
    for n in (most, most - 1, 7104, 1184, 888, 444, 5, 1):
        if n <= most:
            assert all(torch.equal(a, b) for a, b in zip(step(n, scratch), step(n, byte(n)))), n
