"""The largest vocabularies that the token operators accept, on rows that fit the card."""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def test_embedding_of_the_largest_vocabulary():
    import torch
    import paper_2003_11666_b200 as p
    vocab = 2 ** 31 - 1                                            # one column: 4.3 GB
    table = torch.zeros(vocab, 1, device="cuda", dtype=torch.bfloat16)
    rows = torch.tensor([vocab - 1, 0, 2 ** 30], device="cuda")
    table[rows, 0] = torch.tensor([3.0, 2.0, 5.0], device="cuda", dtype=torch.bfloat16)
    ids = torch.cat([rows, torch.tensor([-1, 7], device="cuda")]).to(torch.int32)
    out = torch.empty(5, 1, device="cuda", dtype=torch.bfloat16)
    p.embed_forward(table, ids, out)
    assert out[:, 0].tolist() == [3.0, 2.0, 5.0, 0.0, 0.0]
    for n in (5, 5000):                                            # sorted by one block, and by several
        many, dout = ids.repeat(n // 5), torch.ones(n, 1, device="cuda", dtype=torch.bfloat16)
        scratch = torch.empty(p.embed_scratch_bytes(n, vocab, 1), device="cuda", dtype=torch.uint8)
        hit = torch.cat([rows, rows.new_tensor([7])])
        table.fill_(9.0)
        p.embed_backward(dout, many, table, scratch)
        assert (table[hit, 0] == n // 5).all() and int(torch.count_nonzero(table)) == 4
        table.zero_()
        table[hit[0], 0] = 1.0
        p.embed_backward(dout, many, table, scratch, accumulate=True)
        # n / 5 + 1 in the first row, to the step of bf16
        assert abs(float(table[hit[0], 0]) - (n // 5 + 1)) <= (n // 5 + 1) * 2.0 ** -8 and (table[hit[1:], 0] == n // 5).all()
        assert int(torch.count_nonzero(table)) == 4


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_log_probabilities_of_the_largest_vocabulary(dtype):
    import torch
    import paper_2003_11666_b200 as p
    vocab = 2 ** 30
    x = torch.zeros(1, vocab, device="cuda", dtype=getattr(torch, dtype))
    x[0, vocab - 1], x[0, 12345], x[0, vocab - 3] = 5.0, -3.0, 1.0
    f = lambda *n: torch.empty(*n, device="cuda")                 # noqa: E731
    logp, lse, entropy, top, ids = f(1), f(1), f(1), f(1, 5), torch.empty(1, 5, device="cuda", dtype=torch.int32)
    tok = torch.tensor([vocab - 1], device="cuda")
    p.logprob_forward(x, tok, logp, entropy=entropy, lse=lse, top_logp=top, top_ids=ids)
    log_z = math.log(vocab - 3 + math.exp(5.0) + math.exp(-3.0) + math.exp(1.0))
    # chains of float32 additions: a warp's lane adds 2^30 / (16 * 8 * 32) numbers to two sums of its own
    tol = 2 ** 17 * U + 32 * U
    assert ids.tolist() == [[vocab - 1, vocab - 3, 0, 1, 2]]
    assert abs(float(lse) - log_z) <= tol and abs(float(logp) - (5.0 - log_z)) <= tol
    for got, value in zip(top[0].tolist(), (5.0, 1.0, 0.0, 0.0, 0.0)):
        assert abs(got - (value - log_z)) <= tol
    # H = log Z - sum p x
    assert abs(float(entropy) - (log_z - (5.0 * math.exp(5.0) - 3.0 * math.exp(-3.0) + math.exp(1.0)) * math.exp(-log_z))) <= 2 * tol * log_z
    d = torch.empty_like(x)
    p.logprob_backward(x, tok, lse, d, g_logp=torch.ones(1, device="cuda"))
    store = 2.0 ** -8 if dtype == "bfloat16" else U
    for at, value in ((0, 0.0), (vocab - 2, 0.0), (vocab - 3, 1.0), (12345, -3.0)):
        want = -math.exp(value - float(lse))
        # log p of size 24: three roundings of numbers below 32, and the exponential's 2^-22
        assert abs(float(d[0, at]) - want) <= -want * (3 * 32 * U + 2.0 ** -22 + store)
    assert abs(float(d[0, -1]) - 1.0) <= store + 2.0 ** -20
