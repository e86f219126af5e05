"""Calls that the token operators refuse, on any machine: sizes, types, strides, NULL pointers, alignment and
overlaps are checked on the host before anything is launched."""
import ctypes as C

import pytest

ARG = -1


@pytest.fixture(scope="module")
def lib():
    from paper_2003_11666_b200 import build
    build.build()
    import paper_2003_11666_b200 as p
    return p.load_library()


def _embed_forward(lib, **change):
    a = dict(table=1 << 20, dtype=1, vocab=100, dim=64, ld=64, ids=1 << 30, id_bytes=8, n=10, scale=1.0, out=1 << 31, ld_out=64, status=None,
             stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return lib.pb_embed_forward(*a.values())


@pytest.mark.parametrize("change", [dict(dtype=3), dict(dtype=-1), dict(id_bytes=2), dict(n=-1), dict(n=1 << 31), dict(vocab=0), dict(dim=0),
                                    dict(ld=63), dict(ld_out=63), dict(table=None), dict(ids=None), dict(out=None), dict(table=(1 << 20) + 1),
                                    dict(out=(1 << 31) + 1), dict(ids=(1 << 30) + 4), dict(status=2), dict(out=(1 << 20) + 128)])
def test_embed_forward_refuses(lib, change):
    assert _embed_forward(lib, **change) == ARG
    assert b"pb_embed_forward" in lib.pb_last_error(None)


def _embed_backward(lib, **change):
    a = dict(dout=1 << 20, dtype=1, ld_dout=64, ids=1 << 30, id_bytes=4, n=10, vocab=100, dim=64, scale=1.0, pad=-1, dtable=1 << 31, dt=0, ld=64,
             acc=0, scratch=1 << 32, nscratch=1 << 20, status=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return lib.pb_embed_backward(*a.values())


@pytest.mark.parametrize("change", [dict(dtype=9), dict(dt=2), dict(dtype=0, dt=1), dict(id_bytes=3), dict(n=-5), dict(vocab=0), dict(dim=1 << 31),
                                    dict(ld=10), dict(ld_dout=10), dict(pad=100), dict(pad=-2), dict(acc=2), dict(dtable=None), dict(dout=None),
                                    dict(ids=None), dict(scratch=None), dict(nscratch=16), dict(scratch=(1 << 32) + 128), dict(dtable=(1 << 31) + 2),
                                    dict(dout=1 << 31), dict(scratch=1 << 31), dict(scratch=1 << 20), dict(status=1)])
def test_embed_backward_refuses(lib, change):
    assert _embed_backward(lib, **change) == ARG
    assert b"pb_embed_backward" in lib.pb_last_error(None)


def test_scratch_of_impossible_sizes_is_refused(lib):
    import paper_2003_11666_b200 as p
    assert lib.pb_embed_scratch_bytes(-1, 10, 10) == 0 and lib.pb_embed_scratch_bytes(10, 0, 10) == 0
    assert lib.pb_embed_scratch_bytes(0, 10, 10) > 0
    with pytest.raises(p.PBError):
        p.embed_scratch_bytes(10, 10, 0)


def _logprob_forward(lib, **change):
    a = dict(logits=1 << 20, dtype=1, rows=4, vocab=100, ld=100, tokens=1 << 30, tb=4, it=1.0, logp=1 << 31, entropy=None, lse=None, k=5,
             top=1 << 32, ids=1 << 33, status=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return lib.pb_logprob_forward(*a.values())


@pytest.mark.parametrize("change", [dict(dtype=3), dict(rows=-1), dict(vocab=0), dict(ld=99), dict(it=0.0), dict(it=-1.0), dict(it=float("nan")),
                                    dict(it=float("inf")), dict(it=1e300), dict(it=1e-300), dict(k=-1), dict(k=33), dict(vocab=4, ld=4), dict(logp=None),
                                    dict(tokens=None), dict(tb=1), dict(logits=None), dict(top=None), dict(ids=None), dict(logits=(1 << 20) + 1),
                                    dict(tokens=(1 << 30) + 2), dict(lse=2), dict(entropy=1), dict(status=3)])
def test_logprob_forward_refuses(lib, change):
    assert _logprob_forward(lib, **change) == ARG
    assert b"pb_logprob_forward" in lib.pb_last_error(None)


def _logprob_backward(lib, **change):
    a = dict(logits=1 << 20, dtype=1, rows=4, vocab=100, ld=100, tokens=1 << 30, tb=8, it=1.0, lse=1 << 31, entropy=1 << 32, gl=1 << 33, gh=1 << 34,
             gz=None, d=1 << 35, ld_d=100, status=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return lib.pb_logprob_backward(*a.values())


@pytest.mark.parametrize("change", [dict(dtype=-2), dict(rows=-1), dict(vocab=0), dict(ld=7), dict(ld_d=99), dict(it=0.0), dict(it=float("nan")),
                                    dict(logits=None), dict(d=None), dict(lse=None), dict(tokens=None), dict(entropy=None), dict(tb=2),
                                    dict(d=(1 << 20) + 200), dict(d=1 << 20, ld_d=101), dict(d=(1 << 35) + 1), dict(gl=2)])
def test_logprob_backward_refuses(lib, change):
    assert _logprob_backward(lib, **change) == ARG
    assert b"pb_logprob_backward" in lib.pb_last_error(None)


def _adamw(lib, table=True, grads=True, n=1, **change):
    from paper_2003_11666_b200.binding import pb_adamw_args, pb_adamw_tensor
    t = dict(w=1 << 20, m=1 << 30, v=1 << 31, m_scale=None, v_scale=None, w_forward=None, n=100, weight_decay=0.1, horizon=0.0)
    a = dict(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, step=1, seed=0, dev_grad_scale=None, dev_lr=None, dev_step=None, grad_dtype=0, forward_dtype=0,
             state_bits=32)
    grad = change.pop("grad", 1 << 32)
    for k, v in change.items():
        (a if k in a else t)["n" if k == "size" else k] = v
    tensors, g, args = (pb_adamw_tensor * 1)(pb_adamw_tensor(*t.values())), (C.c_void_p * 1)(grad), pb_adamw_args(*a.values())
    return lib.pb_adamw_step(tensors if table else None, g if grads else None, n, C.byref(args), None)


@pytest.mark.parametrize("change", [dict(n=-1), dict(table=False), dict(grads=False), dict(state_bits=16), dict(grad_dtype=3), dict(forward_dtype=-1),
                                    dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=float("nan")), dict(lr=-1.0), dict(lr=float("inf")), dict(eps=-1.0),
                                    dict(step=0), dict(size=-1), dict(size=1 << 62), dict(weight_decay=-0.5), dict(horizon=float("inf")), dict(w=None),
                                    dict(m=None), dict(v=None), dict(grad=None), dict(state_bits=8), dict(w=(1 << 20) + 2), dict(grad=(1 << 32) + 2),
                                    dict(m=(1 << 30) + 1), dict(w_forward=3), dict(dev_lr=2), dict(dev_step=4), dict(dev_grad_scale=1)])
def test_adamw_refuses(lib, change):
    assert _adamw(lib, **change) == ARG
    assert b"pb_adamw_step" in lib.pb_last_error(None)


def test_adamw_moments_refuses(lib):
    good = [1 << 20, 1 << 30, 1 << 31, 1 << 32, 100, 1 << 33, 1 << 34, None]
    for at, bad in ((0, None), (1, None), (2, None), (3, None), (4, -1), (1, 2), (5, 1), (6, 2)):
        a = list(good)
        a[at] = bad
        assert lib.pb_adamw_moments(*a) == ARG, (at, bad)
    assert lib.pb_adamw_moments(1 << 20, 1 << 30, 1 << 31, 1 << 32, 100, None, None, None) == ARG


def test_calls_without_work_touch_nothing(lib):
    assert _embed_forward(lib, n=0, table=None, ids=None, out=None) == 0
    assert _embed_backward(lib, n=0, acc=1, dout=None, ids=None, dtable=None, scratch=None, nscratch=0) == 0
    assert _logprob_forward(lib, rows=0, logits=None, tokens=None, logp=None, top=None, ids=None) == 0
    assert _logprob_backward(lib, rows=0, logits=None, d=None, lse=None, tokens=None) == 0
    assert _adamw(lib, n=0, table=False, grads=False) == 0
    assert lib.pb_adamw_moments(None, None, None, None, 0, None, None, None) == 0


def test_tensors_on_the_host_are_refused(lib):
    import paper_2003_11666_b200 as p
    import torch
    x, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: p.embed_forward(x, i, x.clone()), lambda: p.embed_backward(x, i, x.clone(), torch.zeros(256, dtype=torch.uint8)),
                 lambda: p.logprob_forward(x, i, x[:, 0].clone()), lambda: p.logprob_backward(x, i, x[:, 0].clone(), x.clone()),
                 lambda: p.AdamW([x], [x.clone()], [x.clone()]), lambda: p.adamw_moments(x, x, x, x, x, x)):
        with pytest.raises(p.PBError) as e:
            call()
        assert e.value.code == ARG


def test_the_package_does_not_need_torch_to_import():
    import subprocess
    import sys
    code = "import sys; import paper_2003_11666_b200 as p; assert 'torch' not in sys.modules; p.load_library()"
    subprocess.run([sys.executable, "-c", code], check=True)
