"""Rows in which one token is all but sure: its log probability, and the row's entropy, are what is left for the others, to float32's digits of that."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


# rows without the tensor cores, a tile of single blocks, pairs; one tile of tokens, many; a sure token at its first, its last, in the middle
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("rows,vocab,dim", [(1, 5000, 256), (2, 60, 512), (4, 9001, 264), (20, 3001, 16), (200, 3001, 8), (130, 100, 1040)])
@pytest.mark.parametrize("gap", [3.0, 9.0, 14.0, 21.0, 40.0])
def test_what_is_left_for_the_others(gap, rows, vocab, dim, dtype):
    import paper_2003_11666_b200 as p
    g = torch.Generator(device="cuda").manual_seed(rows)
    # logits that every type holds: quarters between -1 and 1; row r's own column (the last one is the others') lifts its token by the gap
    h, w = torch.zeros(rows, dim, device="cuda"), torch.zeros(vocab, dim, device="cuda")
    w[:, 0] = torch.randint(-4, 5, (vocab,), generator=g, device="cuda") / 4
    tok = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    tok[0], tok[-1] = vocab - 1, 0
    h[:, 0] = 1.0
    for k in range(1, 8):                                          # seven tokens have a column that lifts them
        w[tok[(k - 1) % rows], k] += gap
    lifted = torch.arange(rows, device="cuda") % 7
    tok = tok[lifted % rows]
    h[torch.arange(rows, device="cuda"), 1 + lifted % min(rows, 7)] = 1.0
    h, w = h.to(dtype), w.to(dtype)
    logp, entropy, lse = (torch.empty(rows, device="cuda") for _ in range(3))
    p.head_logprob_forward(h, w, torch.empty(p.head_scratch_bytes(h, w), device="cuda", dtype=torch.uint8), tok, logp, entropy=entropy, lse=lse)
    z = h.double() @ w.double().T
    top = z.amax(1, keepdim=True)
    rest = torch.where(z < top, (z - top).exp(), 0.0).sum(1)       # of the others; several tokens may be the largest
    ls = torch.log1p(rest + ((z == top).sum(1) - 1))
    want = z.gather(1, tok[:, None])[:, 0] - top[:, 0] - ls
    prob = (z - top - ls[:, None]).exp()
    ref = ls - (prob * (z - top)).sum(1)
    # An exponent below 64 (in units of log 2) is a product of two roundings and of a factor that is off by U, its power is good to 2^-22, and sums of the others take
    # some 40 roundings in a row (sixteen in a thread, a tree, a thread for each part); above a sixteenth the others are what a sum with the largest leaves: 16 roundings of it.
    rel = 2.0 ** -22 + 3 * U * 64 + 40 * U
    near = torch.where(rest > 0.06, 16 * U * (1 + rest), 0.0)
    far = float((top - z).max()) + 2
    for got, value, tol in ((logp, want, rel * ls + near + U * want.abs()), (entropy, ref, (rel * rest + near) * far + 2 * U * ref + rel * ls)):
        err = (got.double() - value).abs()
        assert bool((err <= tol + 1e-37).all()), (float((err / tol).max()), float(err.max()), float(value.abs().min()))
