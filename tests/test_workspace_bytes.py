"""rk_workspace_bytes, and the descriptor of a measured student, whose constant memory has these bytes in it."""
import ctypes as C
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import measure_job
    return measure_job


def test_refuses_nulls():
    import paper_2408_08586_amd as rk
    n, zeros = C.c_uint64(5), C.create_string_buffer(1 << 16)
    assert rk.load_library().rk_workspace_bytes(C.c_void_p(0), C.byref(n)) == rk.RK_ERR_INVALID_ARG
    assert rk.load_library().rk_workspace_bytes(zeros, C.c_void_p(0)) == rk.RK_ERR_INVALID_ARG
    with pytest.raises(rk.RkError):
        rk.rk_workspace_bytes(C.c_void_p(0))
    assert rk.rk_workspace_bytes(zeros) == 0                # a context that has allocated nothing


def test_the_descriptor_counts_working_buffers_once(example):
    import workloads
    wl = workloads.tiny()
    col = {n: i for i, n in enumerate(workloads.COEF_FIELDS)}
    wl.coef[0, col["hidden"]], wl.ints[0, 0] = 5, 24
    constant = float(wl.coef[0, col["mem_const"]])
    m = dict(forward=10.0, forward_layers=4.0, backward=22.0, backward_layers=9.0, bytes_kept=1 << 24, bytes_layers=1 << 23, bytes_library=1 << 28, params_layers=700, params_rest=100)
    coef, _ = example.descriptor(wl, 0, m, layers=2, seq=3, micro_batch=2)
    # (a float32 constant of up to 2^35 bytes)
    assert constant < 2 ** 35 and float(coef[0, col["mem_const"]]) - constant == pytest.approx((1 << 23) + (1 << 28), abs=2.0 ** 12)


@pytest.mark.gpu
def test_buffers_grow_with_calls(example):
    import torch
    import paper_2408_08586_amd as rk
    ctx = rk.rk_create(0)
    rows, vocab, width = 300, 5000, 64
    f = lambda *s: torch.zeros(*s, device="cuda")
    x, w, label, before = f(rows, width).bfloat16(), f(vocab, width).bfloat16(), torch.zeros(rows, dtype=torch.int32, device="cuda"), rk.rk_workspace_bytes(ctx)
    call = lambda: rk.rk_head_loss_backward(ctx, rk.make_head(), x, w, label, None, None, f(rows), f(rows), f(1), torch.empty_like(x), torch.empty_like(w))
    call()
    after = rk.rk_workspace_bytes(ctx)
    assert after - before >= 2 * rows * vocab               # the logits' gradients of one piece among them
    call()
    assert rk.rk_workspace_bytes(ctx) == after
    rk.rk_sync(ctx)
    rk.rk_destroy(ctx)
    m = example.measure(256, 64, 2, layers=1, experts=4, vocab=500, kept=16, steps=2, head=True)
    assert m["bytes_library"] >= 2 * 128 * 500
