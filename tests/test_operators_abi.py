"""Host-side checks of the training-step operators: struct layouts, and what the entry points refuse.

Every refusal comes before the first call of the GPU's runtime, so a context of zeros that names no device is enough for them.
"""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rk():
    import paper_2408_08586_amd as rk
    if not os.path.exists(rk.LIB_PATH):
        from paper_2408_08586_amd import build
        build.build(verbose=False)
    rk.load_library()
    return rk


STRUCTS = ("rk_matrix", "rk_norm_block", "rk_norm_grads", "rk_router", "rk_distill", "rk_teacher")


def test_struct_layouts_match_the_header(rk, tmp_path):
    lines = []
    for s in STRUCTS:
        lines.append(f'printf("{s} %zu\\n", sizeof({s}));')
        lines += [f'printf("{s}.{f[0]} %zu\\n", offsetof({s}, {f[0]}));' for f in getattr(rk, s)._fields_]
    src, exe = str(tmp_path / "a.c"), str(tmp_path / "a.out")
    with open(src, "w") as f:
        f.write('#include <stdio.h>\n#include "rubick.h"\nint main(void){' + "\n".join(lines) + "return 0;}")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), src, "-o", exe], check=True)
    want = dict(l.split() for l in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines())
    for s in STRUCTS:
        cls = getattr(rk, s)
        assert C.sizeof(cls) == int(want[s])
        for f in cls._fields_:
            assert getattr(cls, f[0]).offset == int(want[f"{s}.{f[0]}"]), (s, f[0])


def test_constants_match_the_header(rk):
    text = open(os.path.join(ROOT, "include", "rubick.h")).read()
    for name in ("RK_F32", "RK_BF16", "RK_F16", "RK_NORM_MAX_WIDTH", "RK_MAX_EXPERTS", "RK_MAX_TOP_K", "RK_MAX_TEACHER_LOGITS"):
        assert int(text.split(f"#define {name} ")[1].split()[0].rstrip("u")) == getattr(rk, name), name
    for name, v in rk.RK_NORM_KINDS.items():
        assert int(text.split(f"#define RK_NORM_{name.upper()} ")[1].split()[0].rstrip("u")) == v


class Caller:
    """Calls with plausible arguments, single ones of them replaced."""
    P = 0x1000                                              # an address that is never followed

    def __init__(self, rk):
        self.rk, self.lib = rk, rk.load_library()
        self.ctx = C.create_string_buffer(1 << 16)
        self.keep = []

    def matrix(self, stride=64, type=None, data=P):
        m = self.rk.rk_matrix(data, stride, self.rk.RK_BF16 if type is None else type)
        self.keep.append(m)
        return C.byref(m)

    def text(self):
        return self.rk.rk_last_error(self.ctx)

    def forward(self, rows=4, width=64, ctx=True, **o):
        P, g = self.P, o.get
        b = self.rk.rk_norm_block(g("post", 1), g("pre", 1), g("post_eps", 1e-6), g("pre_eps", 1e-6), g("scale", 1.0), g("ptype", 1),
                                  g("w1", P), g("b1", None), g("w2", P), g("b2", None), g("gate", P), g("gate_rows", 0), g("gate_stride", 0))
        m = self.matrix
        return self.lib.rk_norm_forward(self.ctx if ctx else None, C.byref(b) if g("block", True) else None, C.c_uint64(rows), C.c_uint32(width),
                                        g("x", m()), g("y", m()), g("x_out", m()), g("u", m()), C.c_void_p(g("stats", P)))

    def backward(self, rows=4, width=64, **o):
        P, g = self.P, o.get
        b = self.rk.rk_norm_block(g("post", 1), g("pre", 1), 1e-6, 1e-6, 1.0, g("ptype", 1), g("w1", P), None, g("w2", P), None, g("gate", P),
                                  g("gate_rows", 0), g("gate_stride", 64))
        grads = self.rk.rk_norm_grads(g("g_w1", P), g("g_b1", None), g("g_w2", P), g("g_b2", None), g("g_gate", P), g("g_stride", 64))
        m = self.matrix
        return self.lib.rk_norm_backward(self.ctx, C.byref(b), C.c_uint64(rows), C.c_uint32(width), g("x", m()), g("y", m()),
                                         C.c_void_p(g("stats", P)), g("dxo", m()), g("du", m()), g("dx", m()), g("dy", m()), C.byref(grads))

    def route(self, back=False, n=4, e=16, k=2, renorm=1, group=0, **o):
        P, g = self.P, o.get
        r = self.rk.rk_router(e, k, renorm, group)
        p = lambda name: C.c_void_p(g(name, P))
        head = (self.ctx, C.byref(r) if g("router", True) else None, C.c_uint64(n), g("logits", self.matrix()))
        if back:
            return self.lib.rk_route_backward(*head, p("expert"), p("lse"), p("counts"), p("tokens"), p("d_loss"), p("d_weight"), g("d_logits", self.matrix()))
        return self.lib.rk_route_forward(*head, p("mask"), p("expert"), p("weight"), p("lse"), p("counts"), p("prob_sum"), p("tokens"), p("loss"))

    def distill(self, way="loss", rows=4, vocab=64, tau=1.0, kd=0.5, ce=0.5, k=8, **o):
        P, g = self.P, o.get
        d = self.rk.rk_distill(tau, kd, ce)
        tl = self.rk.rk_matrix(g("t_data", P), g("t_stride", 8), g("t_type", 0))
        self.keep.append(tl)
        t = self.rk.rk_teacher(C.cast(C.byref(tl), C.c_void_p) if g("teacher", True) else None, g("index", P), k, g("label", P), g("weight", P))
        p = lambda name: C.c_void_p(g(name, P))
        head = (self.ctx, C.byref(d) if g("d", True) else None, C.c_uint64(rows), C.c_uint32(vocab), g("student", self.matrix()), C.byref(t) if g("t", True) else None)
        if way == "loss":
            return self.lib.rk_distill_loss(*head, p("loss"), p("lse"), p("total"))
        if way == "backward":
            return self.lib.rk_distill_backward(*head, p("lse"), p("d_total"), g("d_student", self.matrix()))
        return self.lib.rk_distill_loss_backward(*head, p("d_total"), p("loss"), p("lse"), p("total"), g("d_student", self.matrix()))


@pytest.fixture
def call(rk):
    return Caller(rk)


def test_null_contexts(rk):
    for name in ("rk_norm_forward", "rk_norm_backward", "rk_route_forward", "rk_route_backward", "rk_distill_loss", "rk_distill_backward",
                 "rk_distill_loss_backward"):
        assert getattr(rk.load_library(), name)(*[C.c_void_p(0)] * 13) == rk.RK_ERR_INVALID_ARG


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("bad", [
    dict(block=False), dict(post=3), dict(pre=7), dict(post_eps=-1.0), dict(pre_eps=NAN), dict(scale=INF), dict(scale=NAN), dict(ptype=3), dict(ptype=2),
    dict(post=0), dict(pre=0), dict(pre=0, w2=None), dict(y=None), dict(y=None, post=0, w1=None), dict(x=None), dict(u=None), dict(width=0), dict(stats=None),
    dict(stats=0x1004), dict(w1=0x1001), dict(gate=0x1001), dict(gate=None, gate_rows=2), dict(gate_rows=2, gate_stride=63), dict(width=65),
    dict(u=None, x_out=None, pre=0, w2=None)])
def test_norm_forward_refuses(call, rk, bad):
    assert call.forward(**bad) == rk.RK_ERR_INVALID_ARG and call.text()


def test_norm_forward_refuses_matrices(call, rk):
    m = call.matrix
    for name in ("x", "y", "x_out", "u"):
        for bad in (m(stride=63), m(data=None), m(data=0x1001), m(type=3), m(stride=1 << 41)):
            assert call.forward(**{name: bad}) == rk.RK_ERR_INVALID_ARG, name
    assert call.forward(u=m(type=rk.RK_F16)) == rk.RK_ERR_INVALID_ARG
    assert call.forward(x=m(type=rk.RK_F32)) == rk.RK_ERR_INVALID_ARG                       # x_out is not float32
    assert call.forward(x=m(type=rk.RK_F16), x_out=m(type=rk.RK_F16)) == rk.RK_ERR_INVALID_ARG
    wide = m(stride=40000)
    assert call.forward(width=32769, x=wide, y=wide, x_out=wide, u=wide) == rk.RK_ERR_UNSUPPORTED
    assert call.forward(rows=1 << 31) == rk.RK_ERR_UNSUPPORTED
    assert call.forward(rows=0) == rk.RK_OK                                                 # nothing to do, nothing launched


@pytest.mark.parametrize("bad", [
    dict(du=None), dict(dy=None), dict(y=None, post=0, w1=None, gate=None), dict(dx=None), dict(pre=0, w2=None, du=None, dxo=None), dict(g_b1=0x1000),
    dict(g_w1=0x1002), dict(gate=None), dict(gate_rows=2, g_stride=63), dict(stats=None)])
def test_norm_backward_refuses(call, rk, bad):
    assert call.backward(**bad) == rk.RK_ERR_INVALID_ARG and call.text()


def test_norm_backward_refuses_matrices(call, rk):
    m = call.matrix
    for name in ("x", "y", "dxo", "du", "dx", "dy"):
        for bad in (m(stride=63), m(data=None), m(data=0x1001), m(type=3), m(type=rk.RK_F16)):
            assert call.backward(**{name: bad}) == rk.RK_ERR_INVALID_ARG, name


@pytest.mark.parametrize("back", [False, True])
def test_route_refuses(call, rk, back):
    m = call.matrix
    for bad in (dict(router=False), dict(e=0), dict(k=0), dict(k=17), dict(renorm=2), dict(logits=m(stride=15)), dict(logits=m(data=None)), dict(logits=m(type=9)),
                dict(logits=None), dict(lse=0x1002), dict(lse=None), dict(expert=None), dict(counts=None), dict(tokens=None)):
        assert call.route(back, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    for bad in ([dict(d_loss=None), dict(d_loss=0x1001), dict(d_weight=0x1003), dict(d_logits=None), dict(d_logits=m(type=rk.RK_F32)), dict(d_logits=m(stride=3))] if back
                else [dict(weight=None), dict(prob_sum=None), dict(loss=None), dict(weight=0x1001)]):
        assert call.route(back, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    wide = m(stride=2000)
    assert call.route(back, e=1025, logits=wide, d_logits=wide) == rk.RK_ERR_UNSUPPORTED
    assert call.route(back, k=33, e=64, d_logits=m()) == rk.RK_ERR_UNSUPPORTED
    assert call.route(back, n=1 << 24) == rk.RK_ERR_UNSUPPORTED


@pytest.mark.parametrize("way", ["loss", "backward", "both"])
def test_distill_refuses(call, rk, way):
    m = call.matrix
    for bad in (dict(d=False), dict(t=False), dict(tau=0.0), dict(tau=-1.0), dict(tau=NAN), dict(tau=INF), dict(kd=-1.0), dict(ce=NAN), dict(kd=INF), dict(kd=0.0, ce=0.0),
                dict(vocab=0), dict(vocab=65), dict(student=None), dict(student=m(data=None)), dict(student=m(type=4)), dict(teacher=False), dict(kd=0.0),
                dict(label=None), dict(ce=0.0), dict(k=0), dict(k=9), dict(t_data=None), dict(t_type=3), dict(index=None), dict(index=0x1001), dict(weight=0x1002),
                dict(label=0x1001), dict(lse=None), dict(lse=0x1001)):
        assert call.distill(way, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    for bad in [dict(loss=None), dict(total=None), dict(total=0x1002)] if way != "backward" else []:
        assert call.distill(way, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    for bad in [dict(d_student=None), dict(d_student=m(type=rk.RK_F16)), dict(d_student=m(stride=63)), dict(d_total=0x1001)] if way != "loss" else []:
        assert call.distill(way, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    assert call.distill(way, k=1025, t_stride=2000) == rk.RK_ERR_UNSUPPORTED
    assert call.distill(way, rows=1 << 31) == rk.RK_ERR_UNSUPPORTED


def test_the_binding_refuses_before_the_library(rk):
    import torch
    with pytest.raises(rk.RkError):
        rk.NormBlock(post="batch")
    block = rk.NormBlock()
    z = lambda *s, **k: torch.zeros(*s, **k)
    for args in ((z(4, 8), z(4, 8), z(4, 8), z(4, 8), z(4, 4)),                 # not on a GPU
                 (z(4), None, z(4), z(4), z(4))):
        with pytest.raises(rk.RkError):
            rk.rk_norm_forward(C.create_string_buffer(1 << 16), block, *args)
    for t in (z(4, 8).t(), z(4), z(4, 8, dtype=torch.float64), z(1, 8).expand(4, 8)):
        with pytest.raises(rk.RkError):
            rk._matrix(t, "t")
    with pytest.raises(rk.RkError):
        rk._plain(z(4, 8, dtype=torch.int64), "t", (4, 8), ("int32",))
    assert rk._matrix(z(4, 12)[:, 2:10], "t").stride == 12
