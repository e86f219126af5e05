"""Log probabilities over the whole range of sizes, masks and temperatures that are accepted, on the GPU against the
float64 oracle, with the tolerances that tests/test_gpu_tokens.py derives."""
import numpy as np
import pytest

from tests.test_gpu_tokens import _logprob_case, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [262145 + 512, 300000, 524287, 600001, 700003])
@pytest.mark.parametrize("kind", ["normal", "ties"])
def test_alternatives_of_float32_rows_with_many_segments(vocab, kind):
    # more maxima than the selection keeps in registers, by rows of one block and of a cluster
    for rows in (1, 3, 300):
        if rows * vocab > 4e7 and kind == "ties":
            continue
        for k in (1, 20) if rows < 300 else (20,):
            torch, p = _torch()
            if rows < 300:
                _logprob_case(rows, vocab, "float32", kind, 1.0, k, offset=rows)
                continue
            x = torch.randn(rows, vocab, device="cuda")
            top, ids = torch.empty(rows, k, device="cuda"), torch.empty(rows, k, dtype=torch.int32, device="cuda")
            p.logprob_forward(x, top_logp=top, top_ids=ids)
            assert torch.equal(ids.long(), torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k])


def test_alternatives_of_a_long_float32_row_that_is_not_finite():
    torch, p = _torch()
    vocab, k = 300000, 20
    x = torch.randn(4, vocab, device="cuda")
    x[0, 7] = float("nan")
    x[1] = -float("inf")
    x[2] = torch.finfo(torch.float32).min
    x[3] = float("nan")
    lse, top, ids = torch.empty(4, device="cuda"), torch.empty(4, k, device="cuda"), torch.empty(4, k, dtype=torch.int32, device="cuda")
    p.logprob_forward(x, lse=lse, top_logp=top, top_ids=ids)
    assert (ids[[0, 1, 3]] == -1).all() and torch.equal(ids[2].cpu(), torch.arange(k, dtype=torch.int32))
    assert top[[0, 3]].isnan().all() and (top[1] == -float("inf")).all() and lse[[0, 3]].isnan().all()
    # equal logits: each has the logarithm of 1 / vocab, rounded once
    assert np.abs(top[2].double().cpu().numpy() + np.log(vocab)).max() <= np.log(vocab) * 2.0 ** -22
