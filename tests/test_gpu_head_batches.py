"""A scratch laid out for a program's largest batch serves its shorter ones."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("most,vocab,dim,pad", [(64, 1000, 512, 0), (150, 9000, 256, 0), (300, 2000, 136, 0), (70, 1000, 514, 3), (8300, 9001, 16, 0)])
def test_shorter_batches_in_the_scratch_of_the_longest(most, vocab, dim, pad, dtype):
    import paper_2003_11666_b200 as p
    g = torch.Generator(device="cuda").manual_seed(most)
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    wide = rand(most, dim + pad).to(dtype)
    h, w = wide[:, :dim], (rand(vocab, dim) * 0.1).to(dtype)
    tok, gl = torch.randint(0, vocab, (most,), generator=g, device="cuda"), rand(most)
    byte = lambda *a: torch.empty(p.head_scratch_bytes(*a), device="cuda", dtype=torch.uint8)      # noqa: E731
    forward, backward = byte(h, w), byte(h, w, True)

    def step(n, f, b):
        logp, lse, dh, dw = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, dim, device="cuda", dtype=dtype), torch.empty_like(w)
        p.head_logprob_forward(h[:n], w, f, tok[:n], logp, lse=lse)
        p.head_logprob_backward(h[:n], w, b, tok[:n], lse, dh, dw, g_logp=gl[:n])
        return logp, lse, dh, dw
    for n in (most, most - 1, 200, 129, 128, 64, 5, 4, 3, 2, 1):
        if n <= most:
            own = step(n, byte(h[:n], w), byte(h[:n], w, True))
            assert all(torch.equal(a, b) for a, b in zip(step(n, forward, backward), own)), n
