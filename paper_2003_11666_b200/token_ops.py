"""Token operators and the AdamW step on torch tensors: argument marshalling only.

Each function has the name and meaning of the C entry point it calls (include/pb.h) and
works on CUDA tensors that the caller owns, on the current device.  Outputs are written in
place; nothing is allocated, computed or synchronised here.  Calls run on torch's current
stream, like the torch operations that make and use their tensors; `stream`, a cudaStream_t as
an integer (0: the legacy default stream), names another one.  Arguments that do not fit raise
PBError with code -1 before anything is launched.
"""
import ctypes as C
import struct

import torch

from .binding import PBError, load_library, pb_adamw_args, pb_adamw_tensor

_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_ID_BYTES = {torch.int64: 8, torch.int32: 4}
_ARG = -1


def _refuse(who, text):
    raise PBError(_ARG, "%s: %s" % (who, text))


_lib = load_library()


def _check(rc):
    if rc != 0:
        raise PBError(rc, _lib.pb_last_error(None).decode())


# The current device, and its current stream as an integer: what torch.cuda.current_device() and current_stream() ask,
# without their other work (a CUDA tensor is at hand, so CUDA is up).
_current_device, _current = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream

_address, _numel, _get_device, _is_contiguous = torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.get_device, torch.Tensor.is_contiguous

_OFF_DEVICE = "every tensor must be a CUDA tensor on the current device"
_NOT_THAT = "an argument is not what it has to be: tensors on the current device, and numbers"
_MISFITS = (AttributeError, TypeError, OverflowError, struct.error, C.ArgumentError)      # what such an argument raises on its way to the C call


def _on_device(who, device, *tensors):
    """Every tensor given lives on `device`, the current one."""
    try:
        for t in tensors:
            if t is not None and t.get_device() != device:
                _refuse(who, _OFF_DEVICE)
    except AttributeError:
        _refuse(who, _OFF_DEVICE)


def _device(who, t):
    d = t.get_device() if isinstance(t, torch.Tensor) else -1
    if d < 0 or d != _current_device():
        _refuse(who, _OFF_DEVICE)
    return d


def _rows(who, name, t):
    """(rows, columns, row stride) of a matrix whose rows are dense."""
    if t is None:
        _refuse(who, "%s is needed" % name)
    shape = t.shape
    if len(shape) != 2 or t.dtype not in _DTYPE:
        _refuse(who, "%s must be a matrix of float32, bfloat16 or float16" % name)
    rows, cols = shape
    stride, step = t.stride()
    if step != 1 and cols > 1:
        _refuse(who, "%s must have dense rows" % name)
    return rows, cols, stride if rows > 1 else cols


def _vector(who, name, t, n, dtype=torch.float32):
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        _refuse(who, "%s must be a dense %s tensor of %d elements" % (name, dtype, n))
    return t.data_ptr()


def _ids(who, name, t):
    if t is None:
        _refuse(who, "%s is needed" % name)
    size = _ID_BYTES.get(t.dtype)
    if size is None or not t.is_contiguous():
        _refuse(who, "%s must be a dense int32 or int64 tensor" % name)
    return t.data_ptr(), size


def _status(who, t):
    return None if t is None else _vector(who, "status", t, 1, torch.int32)


def embed_forward(table, ids, out, scale=1.0, status=None, stream=None):
    """pb_embed_forward: out[t] = scale * table[ids[t]].  out: [n_tokens, dim], rows may be strided."""
    who = "embed_forward"
    d = _device(who, table)
    _on_device(who, d, ids, out, status)
    vocab, dim, ld = _rows(who, "table", table)
    p, size = _ids(who, "ids", ids)
    rows, cols, ld_out = _rows(who, "out", out)
    if rows != ids.numel() or cols != dim or out.dtype is not table.dtype:
        _refuse(who, "out must be [number of ids, dim] of the table's type")
    _check(_lib.pb_embed_forward(table.data_ptr(), _DTYPE[table.dtype], vocab, dim, ld, p, size, rows, scale,
                                           out.data_ptr(), ld_out, _status(who, status), _current(d) if stream is None else stream))


def embed_scratch_bytes(n_tokens, vocab, dim):
    """pb_embed_scratch_bytes: bytes of scratch that embed_backward needs for these sizes."""
    n = _lib.pb_embed_scratch_bytes(int(n_tokens), int(vocab), int(dim))
    if n == 0:
        _refuse("embed_scratch_bytes", "sizes out of range")
    return n


def embed_backward(dout, ids, dtable, scratch, scale=1.0, padding_idx=-1, accumulate=False, status=None, stream=None):
    """pb_embed_backward: dtable[v] (+)= scale * sum of dout[t] over ids[t] == v.  scratch: uint8 tensor of
    embed_scratch_bytes(...) bytes."""
    who = "embed_backward"
    d = _device(who, dtable)
    _on_device(who, d, dout, ids, scratch, status)
    vocab, dim, ld = _rows(who, "dtable", dtable)
    rows, cols, ld_dout = _rows(who, "dout", dout)
    p, size = _ids(who, "ids", ids)
    if rows != ids.numel() or cols != dim:
        _refuse(who, "dout must be [number of ids, dim]")
    if scratch is None or scratch.dtype is not torch.uint8 or not scratch.is_contiguous():
        _refuse(who, "scratch must be a dense uint8 tensor")
    _check(_lib.pb_embed_backward(dout.data_ptr(), _DTYPE[dout.dtype], ld_dout, p, size, rows, vocab, dim, scale,
                                            padding_idx, dtable.data_ptr(), _DTYPE[dtable.dtype], ld, 1 if accumulate else 0,
                                            scratch.data_ptr(), scratch.numel(), _status(who, status), _current(d) if stream is None else stream))


def logprob_forward(logits, tokens=None, logp=None, entropy=None, lse=None, top_logp=None, top_ids=None, inv_temperature=1.0,
                    status=None, stream=None):
    """pb_logprob_forward: log probabilities of `tokens`, entropies, logsumexps and top alternatives of rows of logits."""
    who = "logprob_forward"
    d = _device(who, logits)
    _on_device(who, d, tokens, logp, entropy, lse, top_logp, top_ids, status)
    rows, vocab, ld = _rows(who, "logits", logits)
    p, size = None, 4
    if tokens is not None:
        p, size = _ids(who, "tokens", tokens)
        if tokens.numel() != rows:
            _refuse(who, "tokens must hold one id per row")
    if (tokens is None) != (logp is None):
        _refuse(who, "logp and tokens go together")
    k = 0
    if (top_logp is None) != (top_ids is None):
        _refuse(who, "top_logp and top_ids go together")
    if top_ids is not None:
        if top_ids.dim() != 2 or top_ids.shape[0] != rows:
            _refuse(who, "top_ids must be [rows, top_k]")
        k = top_ids.shape[1]
    _check(_lib.pb_logprob_forward(
        logits.data_ptr(), _DTYPE[logits.dtype], rows, vocab, ld, p, size, inv_temperature, _vector(who, "logp", logp, rows),
        _vector(who, "entropy", entropy, rows), _vector(who, "lse", lse, rows), k, _vector(who, "top_logp", top_logp, rows * k),
        _vector(who, "top_ids", top_ids, rows * k, torch.int32), _status(who, status), _current(d) if stream is None else stream))


def logprob_backward(logits, tokens, lse, dlogits, g_logp=None, g_entropy=None, entropy=None, g_lse=None, inv_temperature=1.0,
                     status=None, stream=None):
    """pb_logprob_backward: gradient with respect to the logits (dlogits may be the logits themselves)."""
    who = "logprob_backward"
    d = _device(who, logits)
    _on_device(who, d, tokens, lse, dlogits, g_logp, g_entropy, entropy, g_lse, status)
    rows, vocab, ld = _rows(who, "logits", logits)
    drows, dcols, ld_d = _rows(who, "dlogits", dlogits)
    if (drows, dcols) != (rows, vocab) or dlogits.dtype is not logits.dtype:
        _refuse(who, "dlogits must have the logits' shape and type")
    p, size = None, 4
    if tokens is not None:
        p, size = _ids(who, "tokens", tokens)
        if tokens.numel() != rows:
            _refuse(who, "tokens must hold one id per row")
    _check(_lib.pb_logprob_backward(
        logits.data_ptr(), _DTYPE[logits.dtype], rows, vocab, ld, p, size, inv_temperature, _vector(who, "lse", lse, rows),
        _vector(who, "entropy", entropy, rows), _vector(who, "g_logp", g_logp, rows), _vector(who, "g_entropy", g_entropy, rows),
        _vector(who, "g_lse", g_lse, rows), dlogits.data_ptr(), ld_d, _status(who, status), _current(d) if stream is None else stream))


def _head(who, hidden, weight):
    """Sizes and row strides of the two operands: (rows, vocab, dim, ld_hidden, ld_weight, dtype)."""
    rows, dim, ldh = _rows(who, "hidden", hidden)
    vocab, wdim, ldw = _rows(who, "weight", weight)
    if wdim != dim or weight.dtype is not hidden.dtype:
        _refuse(who, "weight must be [vocab, dim] of the hidden states' type")
    return rows, vocab, dim, ldh, ldw, _DTYPE[hidden.dtype]


def _scratch(who, t):
    if t is None or t.dtype is not torch.uint8 or not t.is_contiguous():
        _refuse(who, "scratch must be a dense uint8 tensor")
    return t.data_ptr(), t.numel()


def head_scratch_bytes(hidden, weight, backward=False):
    """pb_head_scratch_bytes: bytes of scratch that head_logprob_forward (or _backward) needs for these tensors, and for fewer rows of hidden states."""
    who = "head_scratch_bytes"
    if not isinstance(hidden, torch.Tensor) or not isinstance(weight, torch.Tensor):
        _refuse(who, "hidden and weight must be tensors")
    rows, vocab, dim, ldh, ldw, dtype = _head(who, hidden, weight)
    whole = all(t.data_ptr() % 16 == 0 and (n <= 1 or ld * t.element_size() % 16 == 0) for t, n, ld in ((hidden, rows, ldh), (weight, vocab, ldw)))
    n = _lib.pb_head_scratch_bytes(dtype, rows, vocab, dim, int(whole), int(bool(backward)))
    if n == 0:
        _refuse(who, "sizes out of range")
    return n


def head_logprob_forward(hidden, weight, scratch, tokens=None, logp=None, entropy=None, lse=None, inv_temperature=1.0, status=None, stream=None):
    """pb_head_logprob_forward: log probabilities of `tokens`, entropies and logsumexps of the rows of hidden @ weight.T, whose
    logits are not stored.  scratch: uint8 tensor of head_scratch_bytes(hidden, weight) bytes."""
    who = "head_logprob_forward"
    d = _device(who, hidden)
    _on_device(who, d, weight, scratch, tokens, logp, entropy, lse, status)
    rows, vocab, dim, ldh, ldw, dtype = _head(who, hidden, weight)
    p, size = None, 4
    if tokens is not None:
        p, size = _ids(who, "tokens", tokens)
        if tokens.numel() != rows:
            _refuse(who, "tokens must hold one id per row")
    if (tokens is None) != (logp is None):
        _refuse(who, "logp and tokens go together")
    try:
        rc = _lib.pb_head_logprob_forward(
            hidden.data_ptr(), weight.data_ptr(), dtype, rows, vocab, dim, ldh, ldw, p, size, inv_temperature, _vector(who, "logp", logp, rows),
            _vector(who, "entropy", entropy, rows), _vector(who, "lse", lse, rows), *_scratch(who, scratch), _status(who, status),
            _current(d) if stream is None else stream)
    except _MISFITS:
        _refuse(who, _NOT_THAT)
    _check(rc)


def head_logprob_backward(hidden, weight, scratch, tokens, lse, dhidden=None, dweight=None, g_logp=None, g_entropy=None, entropy=None, g_lse=None,
                          inv_temperature=1.0, accumulate=False, status=None, stream=None):
    """pb_head_logprob_backward: gradients with respect to the hidden states and the head.  scratch: uint8 tensor of
    head_scratch_bytes(hidden, weight, backward=True) bytes."""
    who = "head_logprob_backward"
    d = _device(who, hidden)
    _on_device(who, d, weight, scratch, tokens, lse, dhidden, dweight, g_logp, g_entropy, entropy, g_lse, status)
    rows, vocab, dim, ldh, ldw, dtype = _head(who, hidden, weight)
    p, size = None, 4
    if tokens is not None:
        p, size = _ids(who, "tokens", tokens)
        if tokens.numel() != rows:
            _refuse(who, "tokens must hold one id per row")
    ld_dh = ld_dw = dim
    dw_type = dtype
    if dhidden is not None:
        r, c, ld_dh = _rows(who, "dhidden", dhidden)
        if (r, c) != (rows, dim) or dhidden.dtype is not hidden.dtype:
            _refuse(who, "dhidden must have the hidden states' shape and type")
    if dweight is not None:
        r, c, ld_dw = _rows(who, "dweight", dweight)
        if (r, c) != (vocab, dim):
            _refuse(who, "dweight must have the weight's shape")
        dw_type = _DTYPE[dweight.dtype]
    try:
        rc = _lib.pb_head_logprob_backward(
            hidden.data_ptr(), weight.data_ptr(), dtype, rows, vocab, dim, ldh, ldw, p, size, inv_temperature, _vector(who, "lse", lse, rows),
            _vector(who, "entropy", entropy, rows), _vector(who, "g_logp", g_logp, rows), _vector(who, "g_entropy", g_entropy, rows),
            _vector(who, "g_lse", g_lse, rows), None if dhidden is None else dhidden.data_ptr(), ld_dh, None if dweight is None else dweight.data_ptr(), dw_type,
            ld_dw, 1 if accumulate else 0, *_scratch(who, scratch), _status(who, status), _current(d) if stream is None else stream)
    except _MISFITS:
        _refuse(who, _NOT_THAT)
    _check(rc)


# pb_join_args and pb_join_grads in their own order: one call lays all fields out, where setting them one by one takes as long as the launch.
_JOIN_ARGS, _JOIN_GRADS = struct.Struct("@qqiiiffdQqPPqPqPqqPPPqPqPP"), struct.Struct("@PqPqPqPqPqPPii")


def _plane(who, name, t, shape, dtype, device):
    """Address and row stride of a matrix with dense rows."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        if t.get_device() != device:
            _refuse(who, _OFF_DEVICE)
        _refuse(who, "%s must be a matrix of %d x %d of type %s" % (name, *shape, dtype))
    ld, step = t.stride()
    if step != 1 and shape[1] > 1:
        _refuse(who, "%s must have dense rows" % name)
    return t.data_ptr(), ld if shape[0] > 1 else shape[1]


def _line(who, name, t, n, dtype, device):
    """Address of a dense vector that may be absent."""
    if t is None:
        return 0
    if t.get_device() != device:
        _refuse(who, _OFF_DEVICE)
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        _refuse(who, "%s must be a dense %s tensor of %d elements" % (name, dtype, n))
    return t.data_ptr()


def _one_type(who, a, b):
    """Type of two vectors that have one, if they are there."""
    dtype = a.dtype if a is not None else b.dtype if b is not None else torch.float32
    if dtype not in _DTYPE or (a is not None and b is not None and b.dtype is not dtype):
        _refuse(who, "the norms' weights, and their gradients, must be of one type")
    return dtype


def _join_gate(who, gate, rows_per_gate, rows, dim, dtype, device):
    """Address, row stride and rows per row of the gate."""
    per = (rows or 1) if rows_per_gate is None else rows_per_gate
    if per < 1:
        _refuse(who, "rows_per_gate must be at least 1")
    return *_plane(who, "gate", gate, (-(-rows // per), dim), dtype, device), per


def dropout(x, out, p, seed, offset=0, dev_offset=None, stream=None):
    """pb_dropout: out = x / (1 - p) where kept, else 0; of matrices [rows, dim].  The gradient is the same call on out's gradient."""
    who = "dropout"
    d = _device(who, x)
    try:
        shape, dtype = x.shape, x.dtype
        if len(shape) != 2 or dtype not in _DTYPE:
            _refuse(who, "x must be a matrix of float32, bfloat16 or float16")
        px, ld = _plane(who, "x", x, shape, dtype, d)
        po, ld_out = _plane(who, "out", out, shape, dtype, d)
        at = None if dev_offset is None else _line(who, "dev_offset", dev_offset, 1, torch.int64, d)
        if not -1 << 63 <= offset < 1 << 63:                     # ctypes would drop the bits above
            _refuse(who, "offset must be a 64-bit integer")
        rc = _lib.pb_dropout(px, _DTYPE[dtype], shape[0], shape[1], ld, p, seed & 0xFFFFFFFFFFFFFFFF, offset, at, po, ld_out,
                             _current(d) if stream is None else stream)
    except _MISFITS:
        _refuse(who, _NOT_THAT)
    _check(rc)


def join_forward(x, u, y, h=None, pre_weight=None, post_weight=None, gate=None, rows_per_gate=None, rstd_pre=None, rstd_post=None, residual_scale=1.0,
                 eps=1e-6, p=0.0, seed=0, offset=0, dev_offset=None, stream=None):
    """pb_join_forward: y = residual_scale * x + dropout(gate * norm(u)), h = norm(y).  A norm is there if its weight is; gate:
    [ceil(rows / rows_per_gate), dim] (rows_per_gate None: one row for all)."""
    who = "join_forward"
    d = _device(who, x)
    try:
        shape, of_stream, dtype, f32 = u.shape, x.dtype, u.dtype, torch.float32
        if len(shape) != 2 or of_stream not in _DTYPE or dtype not in _DTYPE:
            _refuse(who, "x and u must be matrices of float32, bfloat16 or float16")
        rows, dim = shape
        weights = _one_type(who, post_weight, pre_weight)
        px, ld_x = _plane(who, "x", x, shape, of_stream, d)
        pu, ld_u = _plane(who, "u", u, shape, dtype, d)
        py, ld_y = _plane(who, "y", y, shape, of_stream, d)
        ph, ld_h = (0, dim) if h is None else _plane(who, "h", h, shape, dtype, d)
        pg, ld_g, per = (0, dim, 1) if gate is None else _join_gate(who, gate, rows_per_gate, rows, dim, dtype, d)
        args = _JOIN_ARGS.pack(
            rows, dim, _DTYPE[dtype], _DTYPE[of_stream], _DTYPE[weights], residual_scale, eps, p, seed & 0xFFFFFFFFFFFFFFFF, offset,
            0 if dev_offset is None else _line(who, "dev_offset", dev_offset, 1, torch.int64, d), px, ld_x, pu, ld_u, pg, ld_g, per,
            _line(who, "post_weight", post_weight, dim, weights, d), _line(who, "pre_weight", pre_weight, dim, weights, d), py, ld_y, ph, ld_h,
            _line(who, "rstd_post", rstd_post, rows, f32, d), _line(who, "rstd_pre", rstd_pre, rows, f32, d))
        rc = _lib.pb_join_forward(args, _current(d) if stream is None else stream)
    except _MISFITS:
        _refuse(who, _NOT_THAT)
    _check(rc)


def join_scratch_bytes(rows, dim, rows_per_gate=0):
    """pb_join_scratch_bytes: bytes of scratch that join_backward needs for these sizes, and for fewer rows (rows_per_gate 0: no gate)."""
    n = _lib.pb_join_scratch_bytes(int(rows), int(dim), int(rows_per_gate))
    if n == 0:
        _refuse("join_scratch_bytes", "sizes out of range")
    return n


def join_backward(y, u, dx, du, scratch, dy=None, dh=None, pre_weight=None, post_weight=None, gate=None, rows_per_gate=None, rstd_pre=None, rstd_post=None,
                  dpre_weight=None, dpost_weight=None, dgate=None, residual_scale=1.0, p=0.0, seed=0, offset=0, dev_offset=None, stream=None):
    """pb_join_backward: gradients of a join_forward call with the same settings, from its y, u and rstds.  scratch: uint8 tensor of
    join_scratch_bytes(...) bytes; y may be None without dh, dx if it is not wanted."""
    who = "join_backward"
    d = _device(who, u)
    try:
        shape, dtype, f32 = u.shape, u.dtype, torch.float32
        of_stream = dy.dtype if dy is not None else y.dtype if y is not None else dx.dtype if dx is not None else dtype
        if len(shape) != 2 or of_stream not in _DTYPE or dtype not in _DTYPE:
            _refuse(who, "u must be a matrix of float32, bfloat16 or float16, and so the residual stream")
        rows, dim = shape
        weights, grads = _one_type(who, post_weight, pre_weight), _one_type(who, dpost_weight, dpre_weight)
        pu, ld_u = _plane(who, "u", u, shape, dtype, d)
        py, ld_y = (0, dim) if y is None else _plane(who, "y", y, shape, of_stream, d)
        pg, ld_g, per = (0, dim, 1) if gate is None else _join_gate(who, gate, rows_per_gate, rows, dim, dtype, d)
        args = _JOIN_ARGS.pack(
            rows, dim, _DTYPE[dtype], _DTYPE[of_stream], _DTYPE[weights], residual_scale, 0.0, p, seed & 0xFFFFFFFFFFFFFFFF, offset,
            0 if dev_offset is None else _line(who, "dev_offset", dev_offset, 1, torch.int64, d), 0, dim, pu, ld_u, pg, ld_g, per,
            _line(who, "post_weight", post_weight, dim, weights, d), _line(who, "pre_weight", pre_weight, dim, weights, d), py, ld_y, 0, dim,
            _line(who, "rstd_post", rstd_post, rows, f32, d), _line(who, "rstd_pre", rstd_pre, rows, f32, d))
        pdy, ld_dy = (0, dim) if dy is None else _plane(who, "dy", dy, shape, of_stream, d)
        pdh, ld_dh = (0, dim) if dh is None else _plane(who, "dh", dh, shape, dtype, d)
        pdx, ld_dx = (0, dim) if dx is None else _plane(who, "dx", dx, shape, of_stream, d)
        pdu, ld_du = _plane(who, "du", du, shape, dtype, d)
        of_gate, pdg, ld_dg = dtype, 0, dim
        if dgate is not None:
            of_gate = dgate.dtype
            if gate is None or of_gate not in _DTYPE:
                _refuse(who, "dgate goes with a gate, and is of float32 or of its type")
            pdg, ld_dg = _plane(who, "dgate", dgate, gate.shape, of_gate, d)
        out = _JOIN_GRADS.pack(pdy, ld_dy, pdh, ld_dh, pdx, ld_dx, pdu, ld_du, pdg, ld_dg, _line(who, "dpost_weight", dpost_weight, dim, grads, d),
                               _line(who, "dpre_weight", dpre_weight, dim, grads, d), _DTYPE[of_gate], _DTYPE[grads])
        if scratch.get_device() != d:
            _refuse(who, _OFF_DEVICE)
        room, size = _scratch(who, scratch)
        rc = _lib.pb_join_backward(args, out, room, size, _current(d) if stream is None else stream)
    except _MISFITS:
        _refuse(who, _NOT_THAT)
    _check(rc)


def adamw_moments(m, m_scale, v, v_scale, m_out=None, v_out=None, stream=None):
    """pb_adamw_moments: the float32 moments that an 8-bit state stands for."""
    who = "adamw_moments"
    d = _device(who, m)
    _on_device(who, d, m_scale, v, v_scale, m_out, v_out)
    n = m.numel()
    blocks = -(-n // 256)
    _check(_lib.pb_adamw_moments(
        _vector(who, "m", m, n, torch.uint8), _vector(who, "m_scale", m_scale, blocks), _vector(who, "v", v, n, torch.uint8),
        _vector(who, "v_scale", v_scale, blocks), n, _vector(who, "m_out", m_out, n), _vector(who, "v_out", v_out, n),
        _current(d) if stream is None else stream))


class AdamW:
    """pb_adamw_step over a fixed list of tensors: holds the tensors and the table of their addresses.  Weights and
    w_forward may be moved between steps (`w.data = ...`): the table is laid out anew.  The states' memory is held as it
    was given.

    w: float32 weights.  m, v: float32 states, or uint8 ones with m_scale / v_scale (float32, one per 256 elements).
    w_forward: copies of the weights in the forward's type, predicted `horizon` steps ahead, or None.  weight_decay and
    horizon are numbers or one number per tensor.  All tensors are dense, of the caller's, and must not overlap.  One
    thread at a time steps an object.
    """

    def __init__(self, w, m, v, m_scale=None, v_scale=None, w_forward=None, weight_decay=0.0, horizon=0.0):
        who = "AdamW"
        n = len(w)
        lists = [list(x) if x is not None else [None] * n for x in (w, m, v, m_scale, v_scale, w_forward)]
        if any(len(x) != n for x in lists):
            _refuse(who, "the lists must have the same length")
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * n
        ahead = list(horizon) if hasattr(horizon, "__len__") else [horizon] * n
        if len(decay) != n or len(ahead) != n:
            _refuse(who, "weight_decay and horizon are numbers, or one number per tensor")
        for x in lists[1:5]:                                 # names of their own for the states' memory
            x[:] = [t.detach() if isinstance(t, torch.Tensor) else t for t in x]
        self._lists, self._decay, self._ahead = lists, decay, ahead
        self._table = (pb_adamw_tensor * n)()
        self._grads = (C.c_void_p * n)()
        self._args = pb_adamw_args()
        self._args_ref = C.byref(self._args)
        self._may_move = [t for t in lists[0] + lists[5] if t is not None]
        self._lay_out(who)

    def _lay_out(self, who):
        """The table of addresses, and what has to hold of the tensors."""
        lists, n = self._lists, len(self._table)
        self._at = None                                      # until they have been looked at
        for name, x in zip(("w", "m", "v"), lists):
            if any(t is None for t in x):
                _refuse(who, "%s is needed for every tensor" % name)
        self._device = _device(who, lists[0][0]) if n else None
        for x in lists:
            _on_device(who, self._device, *x)
        bits = 8 if n and lists[1][0].dtype is torch.uint8 else 32
        forward = _DTYPE.get(lists[5][0].dtype, -1) if n and lists[5][0] is not None else 0
        self._args.state_bits, self._args.forward_dtype = bits, forward
        self._n = [t.numel() for t in lists[0]]
        state = torch.uint8 if bits == 8 else torch.float32
        spans = []
        for k in range(n):
            tw, tm, tv, ms, vs, tf = (x[k] for x in lists)
            size = self._n[k]
            if (ms is None) != (bits == 32) or (vs is None) != (bits == 32):
                _refuse(who, "8-bit states, and only those, come with scales")
            if (tf is None) != (lists[5][0] is None):
                _refuse(who, "w_forward is given for every tensor or for none")
            blocks = -(-size // 256)
            p = [_vector(who, "w", tw, size), _vector(who, "m", tm, size, state), _vector(who, "v", tv, size, state),
                 _vector(who, "m_scale", ms, blocks), _vector(who, "v_scale", vs, blocks),
                 _vector(who, "w_forward", tf, size, lists[5][0].dtype) if tf is not None else None]
            self._table[k] = pb_adamw_tensor(*p, size, float(self._decay[k]), float(self._ahead[k]))
            spans += [(a, a + t.numel() * t.element_size()) for a, t in zip(p, (tw, tm, tv, ms, vs, tf)) if a and t.numel()]
        if forward < 0:
            _refuse(who, "w_forward must be float32, bfloat16 or float16")
        spans.sort()
        if any(a[1] > b[0] for a, b in zip(spans[:-1], spans[1:])):
            _refuse(who, "two of the tensors overlap")
        self._at = list(map(_address, self._may_move))

    def step(self, grads, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, grad_scale=None, dev_lr=None, dev_step=None, stream=None):
        """One step with `grads`, one tensor per weight, all of one type.  `step` counts from 1."""
        who = "AdamW.step"
        n = len(self._n)
        if len(grads) != n:
            _refuse(who, "one gradient per tensor is needed")
        if n == 0:
            return
        if list(map(_address, self._may_move)) != self._at:
            self._lay_out(who)
        device = self._device
        if device != _current_device():
            _refuse(who, _OFF_DEVICE)
        try:                                                 # a list per property: of many tensors their calls are the time of a step
            dtype = grads[0].dtype
            fits = list(map(_numel, grads)) == self._n and list(map(_get_device, grads)) == [device] * n and \
                all(map(_is_contiguous, grads)) and not any([g.dtype is not dtype for g in grads])
        except (AttributeError, TypeError):                  # None among them, or no tensors
            fits = False
        if not fits:
            _refuse(who, "gradients must be dense CUDA tensors of the weights' sizes and of one type")
        if dtype not in _DTYPE:
            _refuse(who, "gradients must be float32, bfloat16 or float16")
        _on_device(who, device, grad_scale, dev_lr, dev_step)
        self._grads[:] = list(map(_address, grads))
        a = self._args
        a.lr, a.beta1, a.beta2, a.eps, a.step, a.seed, a.grad_dtype = lr, beta1, beta2, eps, step, seed & 0xFFFFFFFFFFFFFFFF, _DTYPE[dtype]
        a.dev_grad_scale = None if grad_scale is None else _vector(who, "grad_scale", grad_scale, 1)
        a.dev_lr = None if dev_lr is None else _vector(who, "dev_lr", dev_lr, 1)
        a.dev_step = None if dev_step is None else _vector(who, "dev_step", dev_step, 1, torch.int64)
        _check(_lib.pb_adamw_step(self._table, self._grads, n, self._args_ref, _current(device) if stream is None else stream))
