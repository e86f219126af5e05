"""Log probabilities of a few rows, which run without the tensor cores where their rows start on 16 bytes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _values(h, w, tok):
    import paper_2003_11666_b200 as p
    out = [torch.empty(h.shape[0], device="cuda") for _ in range(3)]
    sc = torch.empty(p.head_scratch_bytes(h, w), device="cuda", dtype=torch.uint8)
    p.head_logprob_forward(h, w, sc, tok, out[0], entropy=out[1], lse=out[2])
    return out


# row strides of 4 and 8 floats (of 8 halves): the same sums as of rows without a gap
@pytest.mark.parametrize("dtype,pads", [(torch.float32, (4, 8, 12)), (torch.bfloat16, (8, 16)), (torch.float16, (8, 24))], ids=str)
@pytest.mark.parametrize("rows", [1, 2, 3, 4])
def test_rows_on_16_bytes_are_summed_alike(rows, dtype, pads):
    g = torch.Generator(device="cuda").manual_seed(rows)
    h, w = (torch.randn(n, 1024, generator=g, device="cuda").to(dtype) for n in (rows, 777))
    tok = torch.randint(0, 777, (rows,), generator=g, device="cuda")
    ref = _values(h, w, tok)
    for pad in pads:
        a, b = (torch.zeros(t.shape[0], 1024 + pad, device="cuda", dtype=dtype)[:, :1024].copy_(t) for t in (h, w))
        assert all(torch.equal(x, y) for x, y in zip(_values(a, b, tok), ref)), pad
    # rows of 4 floats more than a multiple of 8
    if dtype is torch.float32:
        a, b = h[:, :1020].contiguous(), w[:, :1020].contiguous()
        ref = _values(h[:, :1020], w[:, :1020], tok)               # a stride of 1024
        assert all(torch.equal(x, y) for x, y in zip(_values(a, b, tok), ref))
