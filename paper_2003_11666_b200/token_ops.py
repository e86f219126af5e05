"""Token operators and the AdamW step on torch tensors: argument marshalling only.

Each function has the name and meaning of the C entry point it calls (include/pb.h) and
works on CUDA tensors that the caller owns, on the current device.  Outputs are written in
place; nothing is allocated, computed or synchronised here.  Calls run on torch's current
stream, like the torch operations that make and use their tensors; `stream`, a cudaStream_t as
an integer (0: the legacy default stream), names another one.  Arguments that do not fit raise
PBError with code -1 before anything is launched.
"""
import ctypes as C

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
