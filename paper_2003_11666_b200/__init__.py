"""B200-native Pipelined Backpropagation engine (CUDA library + thin binding).

`PB` wraps one engine handle; see include/pb.h for the meaning of each call.
The package never computes on the CPU: without the built shared library the
binding raises.
"""
from .binding import PB, PBError, mlp_run_static, split_plan, bench_l2_bandwidth, bench_fp32_fma, PB_SC, PB_LWP, PB_LWP_WFORM, PB_CONV_BF16, PB_WEIGHT_STASH, load_library, LIB_PATH, EXPORTS

# The token operators take torch tensors; torch is imported when one of them is first used.
_TOKEN_OPS = ("AdamW", "adamw_moments", "embed_backward", "embed_forward", "embed_scratch_bytes", "logprob_backward", "logprob_forward")


def __getattr__(name):
    if name in _TOKEN_OPS:
        from . import token_ops
        globals().update({n: getattr(token_ops, n) for n in _TOKEN_OPS})
        return globals()[name]
    raise AttributeError("module %r has no attribute %r" % (__name__, name))


__all__ = ["PB", "PBError", "mlp_run_static", "split_plan", "bench_l2_bandwidth", "bench_fp32_fma", "PB_SC", "PB_LWP", "PB_LWP_WFORM", "PB_CONV_BF16", "PB_WEIGHT_STASH", "load_library",
           "LIB_PATH", "EXPORTS", *_TOKEN_OPS]
