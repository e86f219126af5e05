"""Embedding gradients added to what the table's gradient already holds, on the GPU: float32 numbers below 2^-126."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,vocab,dim,ld", [(3, 10, 8, 8), (40, 10, 5, 5), (3000, 70, 72, 72), (3000, 2, 33, 40), (5000, 300, 64, 64)])
def test_subnormal_sums_and_entries_are_kept(n, vocab, dim, ld):
    # multiples of 2^-140 far below 2^24 of them: every float32 sum is exact, in any order
    import torch
    import paper_2003_11666_b200 as p
    rng = np.random.default_rng(n)
    step = 2.0 ** -140
    ids = rng.integers(0, vocab, n)
    x, start = rng.integers(-5, 6, (n, dim)), rng.integers(-9, 10, (vocab, dim))
    ref = start.copy()
    np.add.at(ref, ids, x)
    table = torch.zeros(vocab, ld, device="cuda")[:, :dim]
    table.copy_(torch.tensor(start * step, dtype=torch.float32))
    dout = torch.tensor(x * step, dtype=torch.float32).cuda()
    scratch = torch.empty(p.embed_scratch_bytes(n, vocab, dim), dtype=torch.uint8, device="cuda")
    p.embed_backward(dout, torch.tensor(ids, device="cuda"), table, scratch, accumulate=True)
    np.testing.assert_array_equal(table.cpu().numpy().astype(np.float64) / step, ref)
    # and written over what is there
    p.embed_backward(dout, torch.tensor(ids, device="cuda"), table, scratch)
    ref = np.zeros_like(start)
    np.add.at(ref, ids, x)
    np.testing.assert_array_equal(table.cpu().numpy().astype(np.float64) / step, ref)
