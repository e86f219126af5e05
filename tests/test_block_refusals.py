"""Calls that the head, join and dropout operators refuse, on any machine: everything here is checked on the host before
anything is launched."""
import ctypes as C

import pytest

from tests.test_token_refusals import ARG, lib  # noqa: F401

MB = 1 << 20


def _head_forward(lib, **change):
    a = dict(hidden=1 << 30, weight=1 << 32, dtype=1, rows=10, vocab=100, dim=64, ldh=64, ldw=64, tokens=1 << 34, tb=4, it=1.0, logp=1 << 35, entropy=None,
             lse=None, scratch=1 << 36, nscratch=16 * MB, status=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return lib.pb_head_logprob_forward(*a.values())


@pytest.mark.parametrize("change", [dict(dtype=3), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(dim=0),
                                    dict(dim=(1 << 20) + 1, ldh=1 << 21, ldw=1 << 21), dict(ldh=63), dict(ldw=63), dict(ldw=1 << 37), dict(it=0.0),
                                    dict(it=-1.0), dict(it=float("nan")), dict(it=float("inf")), dict(it=1e39), dict(it=1e-50), dict(logp=None),
                                    dict(tokens=None), dict(tb=2), dict(hidden=None), dict(weight=None), dict(scratch=None), dict(hidden=(1 << 30) + 1),
                                    dict(tokens=(1 << 34) + 2), dict(tokens=(1 << 34) + 4, tb=8), dict(logp=(1 << 35) + 2), dict(lse=2), dict(entropy=1),
                                    dict(status=3), dict(scratch=(1 << 36) + 128), dict(nscratch=100), dict(scratch=(1 << 30) - 256), dict(scratch=1 << 32),
                                    dict(scratch=1 << 34), dict(scratch=1 << 35), dict(lse=(1 << 36) + 400), dict(status=(1 << 36) + 4096)])
def test_head_forward_refuses(lib, change):       # noqa: F811
    assert _head_forward(lib, **change) == ARG
    assert b"pb_head_logprob_forward" in lib.pb_last_error(None)


def _head_backward(lib, **change):
    a = dict(hidden=1 << 30, weight=1 << 32, dtype=1, rows=10, vocab=100, dim=64, ldh=64, ldw=64, tokens=1 << 34, tb=4, it=1.0, lse=1 << 35, entropy=1 << 37,
             gl=1 << 38, ge=1 << 39, gz=None, dh=1 << 40, lddh=64, dw=1 << 41, dwt=0, lddw=64, acc=0, scratch=1 << 36, nscratch=16 * MB, status=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return lib.pb_head_logprob_backward(*a.values())


@pytest.mark.parametrize("change", [dict(dtype=-1), dict(rows=-1), dict(vocab=0), dict(dim=0), dict(ldh=1), dict(ldw=1), dict(it=0.0), dict(lddh=63),
                                    dict(lddw=63), dict(dwt=2), dict(dwt=5), dict(dtype=0, dwt=1), dict(acc=2), dict(dh=None, dw=None), dict(lse=None),
                                    dict(tokens=None), dict(entropy=None), dict(tb=1), dict(hidden=None), dict(weight=None), dict(scratch=None),
                                    dict(scratch=(1 << 36) + 64), dict(nscratch=1000), dict(dh=(1 << 40) + 1), dict(dw=(1 << 41) + 2), dict(gl=2), dict(gz=2),
                                    dict(lse=(1 << 35) + 1), dict(status=1), dict(dh=1 << 30), dict(dh=1 << 32), dict(dw=1 << 32), dict(dw=1 << 40),
                                    dict(dh=1 << 36), dict(dw=(1 << 38) - 64), dict(scratch=1 << 39), dict(status=1 << 40), dict(status=1 << 35),
                                    dict(dh=(1 << 34) - 128), dict(rows=0, dw=(1 << 41) + 2)])
def test_head_backward_refuses(lib, change):      # noqa: F811
    assert _head_backward(lib, **change) == ARG
    assert b"pb_head_logprob_backward" in lib.pb_last_error(None)


def test_head_scratch(lib):                       # noqa: F811
    n = lib.pb_head_scratch_bytes
    for bad in ((3, 1, 10, 10), (1, -1, 10, 10), (1, 1 << 25, 10, 10), (1, 1, 0, 10), (1, 1, 10, 0)):
        assert n(*bad, 1, 0) == 0 and n(*bad, 1, 1) == 0
    assert n(1, 0, 10, 10, 1, 0) > 0
    # not a matrix of logits: a gigabyte of them in bf16, a quarter of that in the backward and a fraction in the forward
    logits = 4096 * 131072 * 2
    assert n(1, 4096, 131072, 4096, 1, 0) < logits // 20
    assert n(1, 4096, 131072, 4096, 1, 1) < logits // 2
    assert n(1, 4096, 131072, 4096, 0, 0) > n(1, 4096, 131072, 4096, 1, 0)
    assert n(0, 10, 1000, 64, 1, 1) == n(0, 10, 1000, 64, 0, 1)


def _dropout(lib, **change):
    a = dict(x=1 << 30, dtype=1, rows=10, dim=64, ldx=64, p=0.1, seed=1, offset=0, dev=None, out=1 << 31, ldo=64, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return lib.pb_dropout(*a.values())


@pytest.mark.parametrize("change", [dict(dtype=3), dict(rows=-1), dict(dim=-1), dict(dim=1 << 31), dict(ldx=63), dict(ldo=63), dict(p=-0.1), dict(p=1.0),
                                    dict(p=float("nan")), dict(p=1 - 2.0 ** -18), dict(x=None), dict(out=None), dict(x=(1 << 30) + 1), dict(out=(1 << 31) + 1),
                                    dict(dev=4), dict(out=(1 << 30) + 2), dict(out=1 << 30, ldo=65), dict(dev=(1 << 31) + 8)])
def test_dropout_refuses(lib, change):            # noqa: F811
    assert _dropout(lib, **change) == ARG
    assert b"pb_dropout" in lib.pb_last_error(None)


def _join(lib, backward=False, args=True, grads=True, scratch=1 << 50, nscratch=16 * MB, **change):
    from paper_2003_11666_b200.binding import pb_join_args, pb_join_grads
    a = dict(rows=10, dim=64, dtype=1, stream_dtype=0, weight_dtype=0, residual_scale=1.0, eps=1e-6, p=0.1, seed=1, offset=0, dev_offset=None, x=1 << 30, ld_x=64,
             u=1 << 31, ld_u=64, gate=1 << 32, ld_gate=64, rows_per_gate=4, post_weight=1 << 33, pre_weight=1 << 34, y=1 << 35, ld_y=64, h=1 << 36, ld_h=64,
             rstd_post=1 << 37, rstd_pre=1 << 38)
    d = dict(dy=1 << 39, ld_dy=64, dh=1 << 40, ld_dh=64, dx=1 << 41, ld_dx=64, du=1 << 42, ld_du=64, dgate=1 << 43, ld_dgate=64, dpost_weight=1 << 44,
             dpre_weight=1 << 45, dgate_dtype=1, dweight_dtype=0)
    for k, v in change.items():
        assert k in a or k in d, k
        (a if k in a else d)[k] = v
    x, g = pb_join_args(), pb_join_grads()
    for o, v in ((x, a), (g, d)):
        for k, n in v.items():
            setattr(o, k, n)
    if backward:
        return lib.pb_join_backward(C.byref(x) if args else None, C.byref(g) if grads else None, scratch, nscratch, None)
    return lib.pb_join_forward(C.byref(x) if args else None, None)


BOTH = [dict(args=False), dict(dtype=4), dict(stream_dtype=2), dict(weight_dtype=2), dict(stream_dtype=7), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(dim=0),
        dict(dim=16385), dict(rows_per_gate=0), dict(ld_gate=63), dict(residual_scale=float("inf")), dict(eps=-1.0), dict(eps=float("nan")), dict(p=1.0),
        dict(p=-1.0), dict(ld_u=63), dict(u=None), dict(u=(1 << 31) + 1), dict(gate=(1 << 32) + 1), dict(post_weight=(1 << 33) + 2), dict(rstd_pre=2),
        dict(dev_offset=4)]


@pytest.mark.parametrize("change", BOTH + [dict(x=None), dict(y=None), dict(ld_x=63), dict(ld_y=63), dict(ld_h=63), dict(h=None), dict(pre_weight=None),
                                           dict(x=(1 << 30) + 2), dict(h=(1 << 36) + 1), dict(y=(1 << 30) + 4), dict(y=1 << 30, ld_y=65), dict(h=1 << 30),
                                           dict(y=1 << 31), dict(h=(1 << 31) + 2), dict(h=1 << 35), dict(y=1 << 32), dict(h=1 << 34), dict(rstd_pre=1 << 37),
                                           dict(rstd_post=1 << 31), dict(dev_offset=1 << 35)])
def test_join_forward_refuses(lib, change):       # noqa: F811
    assert _join(lib, **change) == ARG
    assert b"pb_join_forward" in lib.pb_last_error(None)


@pytest.mark.parametrize("change", BOTH + [dict(grads=False), dict(scratch=None), dict(scratch=(1 << 50) + 8), dict(nscratch=10), dict(dweight_dtype=2),
                                           dict(dgate_dtype=2), dict(dgate_dtype=-1), dict(ld_du=63), dict(ld_dx=63), dict(ld_dy=63), dict(ld_dh=63),
                                           dict(ld_y=63), dict(ld_dgate=63), dict(gate=None), dict(post_weight=None), dict(dh=None), dict(du=None),
                                           dict(dy=None, dh=None, dpre_weight=None), dict(y=None), dict(pre_weight=None), dict(rstd_pre=None),
                                           dict(rstd_post=None), dict(du=(1 << 42) + 1), dict(dx=(1 << 41) + 2), dict(dgate=(1 << 43) + 1),
                                           dict(dpre_weight=(1 << 45) + 2), dict(dx=1 << 35), dict(du=1 << 31), dict(dx=(1 << 39) + 4),
                                           dict(dx=1 << 39, ld_dx=65), dict(du=1 << 41), dict(dgate=1 << 32), dict(dpre_weight=1 << 44), dict(scratch=1 << 43),
                                           dict(scratch=1 << 35), dict(dpost_weight=1 << 38), dict(dev_offset=1 << 42)])
def test_join_backward_refuses(lib, change):      # noqa: F811
    assert _join(lib, backward=True, **change) == ARG
    assert b"pb_join_backward" in lib.pb_last_error(None)


def test_calls_without_work_touch_nothing(lib):   # noqa: F811
    assert _head_forward(lib, rows=0, hidden=None, weight=None, scratch=None, tokens=None, logp=None) == 0
    assert _head_backward(lib, rows=0, acc=1, hidden=None, scratch=None) == 0
    assert _head_backward(lib, rows=0, dw=None, hidden=None, scratch=None) == 0
    assert _dropout(lib, rows=0, x=None, out=None) == 0 and _dropout(lib, dim=0, x=None, out=None) == 0
    assert _join(lib, rows=0, x=None, u=None, y=None, h=None) == 0
    assert _join(lib, backward=True, rows=0, u=None, scratch=None, dpre_weight=None, dpost_weight=None) == 0
    assert _join(lib, backward=True, rows=0, u=None, scratch=None, dy=None, dh=None, gate=None, dpre_weight=None, dpost_weight=None) == 0
    assert lib.pb_join_scratch_bytes(-1, 10, 0) == 0 and lib.pb_join_scratch_bytes(10, 0, 0) == 0 and lib.pb_join_scratch_bytes(10, 16385, 0) == 0
    assert lib.pb_join_scratch_bytes(0, 10, 0) > 0


def test_tensors_on_the_host_and_impossible_sizes_are_refused(lib):      # noqa: F811
    import paper_2003_11666_b200 as p
    import torch
    x, u8, i = torch.zeros(4, 8), torch.zeros(256, dtype=torch.uint8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: p.head_logprob_forward(x, x.clone(), u8, i, x[:, 0].clone()), lambda: p.head_logprob_backward(x, x.clone(), u8, i, x[:, 0].clone(), x.clone()),
                 lambda: p.join_forward(x, x.clone(), x.clone()), lambda: p.join_backward(x, x.clone(), x.clone(), x.clone(), u8, dy=x.clone()),
                 lambda: p.dropout(x, x.clone(), 0.5, 1), lambda: p.head_scratch_bytes(None, x), lambda: p.head_scratch_bytes(x, x[:, :5]),
                 lambda: p.head_scratch_bytes(x, x.half()), lambda: p.join_scratch_bytes(1, 0)):
        with pytest.raises(p.PBError) as e:
            call()
        assert e.value.code == ARG
    assert p.head_scratch_bytes(x, x) > 0
