"""The packed arguments of the joins lie as the C structures do."""
import ctypes as C


def test_packed_fields_lie_as_the_structures():
    from paper_2003_11666_b200 import token_ops as T
    from paper_2003_11666_b200.binding import pb_join_args, pb_join_grads
    for packer, struct in ((T._JOIN_ARGS, pb_join_args), (T._JOIN_GRADS, pb_join_grads)):
        assert packer.size == C.sizeof(struct)
        values = [float(k) if f[1] in (C.c_float, C.c_double) else k for k, f in enumerate(struct._fields_, 1)]
        got = struct.from_buffer_copy(packer.pack(*values))
        assert [getattr(got, f[0]) for f in struct._fields_] == values
