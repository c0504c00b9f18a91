"""Host-side: what the training-step operators refuse beside test_operators_abi.py, and that their binding leaves the library as it is."""
import ctypes as C

import pytest

from test_operators_abi import call, rk  # noqa: F401  (fixtures)


def test_gates_of_the_gradients(call, rk):
    """Fewer gates than the rows need, a stride that lets gates overlap, more than are counted."""
    P, m = call.P, call.matrix

    def backward(rows, gate_rows, gates, stride):
        b = rk.rk_norm_block(1, 1, 1e-6, 1e-6, 1.0, 1, P, None, P, None, P, gate_rows, 64)
        g = rk.rk_norm_grads(P, None, P, None, P, stride, gates)
        return call.lib.rk_norm_backward(call.ctx, C.byref(b), C.c_uint64(rows), C.c_uint32(64), m(), m(), C.c_void_p(P), m(), m(), m(), m(), C.byref(g))

    for rows, gate_rows, gates, stride in ((9, 4, 2, 64), (8, 4, 1, 64), (3, 4, 2, 63), (0, 4, 3, 63), (9, 4, 3, 63), (9, 4, 1 << 31, 64)):
        assert backward(rows, gate_rows, gates, stride) == rk.RK_ERR_INVALID_ARG and call.text(), (rows, gate_rows, gates, stride)


def test_the_binding_leaves_the_librarys_functions_alone(rk):
    """Argument types that the binding sets are its own: a caller of the C functions finds them as they were, whoever called first."""
    lib = rk.load_library()
    for name in rk._OPERATORS:
        own = rk._operator(name)
        assert own is rk._operator(name) and own.argtypes and own.restype is C.c_int32
        assert getattr(lib, name).argtypes is None
        assert getattr(lib, name)(*[C.c_void_p(0)] * 13) == rk.RK_ERR_INVALID_ARG


def test_groups_that_one_launch_cannot_join(call, rk):
    """300,000 groups of 16 tiles of experts, 1,024 threads each."""
    wide = call.matrix(stride=256)
    assert call.route(n=300000, e=256, group=1, logits=wide) == rk.RK_ERR_UNSUPPORTED and "2^26" in call.text()
    assert call.route(n=(1 << 24) - 1, e=33, group=8, logits=wide) == rk.RK_ERR_UNSUPPORTED
