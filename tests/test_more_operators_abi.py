"""Host-side checks of gated recurrence, dropout and vocabulary head: struct layouts, constants, and what the entry points refuse.

Every refusal comes before the first call of the GPU's runtime, so a context of zeros that names no device is enough for them.
"""
import ctypes as C
import os
import subprocess

import pytest

from test_operators_abi import ROOT, Caller, rk  # noqa: F401  (fixture)

NAN, INF = float("nan"), float("inf")


def test_struct_layouts_match_the_header(rk, tmp_path):
    structs = ("rk_recur", "rk_dropout", "rk_head")
    lines = []
    for s in structs:
        lines.append(f'printf("{s} %zu\\n", sizeof({s}));')
        lines += [f'printf("{s}.{f[0]} %zu\\n", offsetof({s}, {f[0]}));' for f in getattr(rk, s)._fields_]
    src, exe = str(tmp_path / "a.c"), str(tmp_path / "a.out")
    with open(src, "w") as f:
        f.write('#include <stdio.h>\n#include <stddef.h>\n#include "rubick.h"\nint main(void){' + "\n".join(lines) + "return 0;}")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), src, "-o", exe], check=True)
    want = dict(l.split() for l in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines())
    for s in structs:
        cls = getattr(rk, s)
        assert C.sizeof(cls) == int(want[s])
        for f in cls._fields_:
            assert getattr(cls, f[0]).offset == int(want[f"{s}.{f[0]}"]), (s, f[0])
    text = open(os.path.join(ROOT, "include", "rubick.h")).read()
    for name in ("RK_RECUR_MAX_WIDTH", "RK_HEAD_MAX_WIDTH"):
        assert int(text.split(f"#define {name} ")[1].split()[0].rstrip("u")) == getattr(rk, name), name


class MoreCaller(Caller):
    def recur(self, back=False, rows=4, width=64, **o):
        P, g, m = self.P, o.get, self.matrix
        f32 = lambda: m(type=self.rk.RK_F32)
        r = self.rk.rk_recur(g("coupled", 1), g("ptype", 1), g("bias", P), g("offsets", P), g("n_seqs", 3), g("seq_rows", 0))
        head = (self.ctx if g("ctx", True) else None, C.byref(r) if g("recur", True) else None, C.c_uint64(rows), C.c_uint32(width))
        if back:
            return self.lib.rk_recur_backward(*head, g("x", m()), g("z", m()), g("h", m()), g("state_in", f32()), g("dh", m()), g("d_state_out", f32()), g("dx", m()),
                                              g("dz", m()), g("d_state_in", f32()), C.c_void_p(g("d_bias", P)))
        return self.lib.rk_recur_forward(*head, g("x", m()), g("z", m()), g("state_in", f32()), g("h", m()), g("state_out", f32()))

    def dropout(self, back=False, rows=4, width=64, **o):
        P, g, m = self.P, o.get, self.matrix
        d = self.rk.rk_dropout(g("p", 0.5), g("rng", P))
        head = (self.ctx if g("ctx", True) else None, C.byref(d) if g("d", True) else None, C.c_uint64(rows), C.c_uint32(width))
        if back:
            return self.lib.rk_dropout_backward(*head, g("d_out", m()), g("dx", m()))
        return self.lib.rk_dropout_forward(*head, g("x", m()), g("residual", m()), g("out", m()))

    def head(self, way="loss", rows=4, width=64, vocab=100, **o):
        P, g, m = self.P, o.get, self.matrix
        h = self.rk.rk_head(g("scale", 1.0), g("z", 0.0))
        p = lambda name: C.c_void_p(g(name, P))
        head = (self.ctx if g("ctx", True) else None, C.byref(h) if g("h", True) else None, C.c_uint64(rows), C.c_uint32(width), C.c_uint32(vocab), g("x", m()),
                g("weight", m()), p("label"), p("row_weight"))
        if way == "loss":
            return self.lib.rk_head_loss(*head, p("loss"), p("lse"), p("total"))
        if way == "backward":
            return self.lib.rk_head_backward(*head, p("lse"), p("d_total"), g("dx", m()), g("d_weight", m()))
        return self.lib.rk_head_loss_backward(*head, p("d_total"), p("loss"), p("lse"), p("total"), g("dx", m()), g("d_weight", m()))


@pytest.fixture
def call(rk):
    return MoreCaller(rk)


def test_null_contexts(rk):
    for name in ("rk_recur_forward", "rk_recur_backward", "rk_dropout_forward", "rk_dropout_backward", "rk_head_loss", "rk_head_backward", "rk_head_loss_backward"):
        assert getattr(rk.load_library(), name)(*[C.c_void_p(0)] * 15) == rk.RK_ERR_INVALID_ARG


@pytest.mark.parametrize("back", [False, True])
def test_recur_refuses(call, rk, back):
    m = call.matrix
    for bad in (dict(recur=False), dict(coupled=2), dict(ptype=3), dict(bias=0x1001), dict(ptype=0, bias=0x1002), dict(offsets=0x1002), dict(seq_rows=4),
                dict(offsets=None), dict(width=0), dict(width=65), dict(z=None), dict(x=None), dict(h=None)):
        assert call.recur(back, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    for name in ("x", "z", "h") + (("dh", "dx", "dz") if back else ()):
        for bad in (m(stride=63), m(data=None), m(data=0x1001), m(type=3), m(type=rk.RK_F16)):
            assert call.recur(back, **{name: bad}) == rk.RK_ERR_INVALID_ARG, name
    f32 = lambda **k: m(type=rk.RK_F32, **k)
    for name in ("state_in",) + (("d_state_out", "d_state_in") if back else ("state_out",)):
        for bad in (m(), f32(stride=63), f32(data=None), f32(data=0x1002)):
            assert call.recur(back, **{name: bad}) == rk.RK_ERR_INVALID_ARG and call.text(), name
    wide = m(stride=1 << 21)
    assert call.recur(back, width=(1 << 20) + 1, z=wide) == rk.RK_ERR_UNSUPPORTED
    assert call.recur(back, rows=1 << 31) == rk.RK_ERR_UNSUPPORTED
    assert call.recur(back, n_seqs=0x7FFFFFFF) == rk.RK_ERR_UNSUPPORTED
    if back:
        for bad in (dict(dx=None), dict(dz=None), dict(dh=None), dict(d_bias=0x1001), dict(bias=None)):
            assert call.recur(True, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    else:
        assert call.recur(rows=0, n_seqs=0, offsets=call.P) == rk.RK_OK       # nothing to do, nothing launched


@pytest.mark.parametrize("back", [False, True])
def test_dropout_refuses(call, rk, back):
    m = call.matrix
    for bad in (dict(d=False), dict(p=-0.1), dict(p=1.5), dict(p=NAN), dict(rng=None), dict(rng=0x1004), dict(width=0), dict(width=65)):
        assert call.dropout(back, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    for name in ("d_out", "dx") if back else ("x", "residual", "out"):
        for bad in (m(stride=63), m(data=None), m(data=0x1001), m(type=3), m(type=rk.RK_F16)):
            assert call.dropout(back, **{name: bad}) == rk.RK_ERR_INVALID_ARG, name
    for bad in (dict(d_out=None), dict(dx=None), dict(dx=m(type=rk.RK_F32))) if back else (dict(x=None), dict(out=None), dict(x=m(type=rk.RK_F32)),
                                                                                         dict(out=m(type=rk.RK_F32)), dict(residual=m(type=rk.RK_F32))):
        assert call.dropout(back, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    wide = m(stride=1 << 29)
    assert call.dropout(back, width=(1 << 28) + 1, x=wide, residual=wide, out=wide, d_out=wide, dx=wide) == rk.RK_ERR_UNSUPPORTED
    assert call.dropout(back, rows=1 << 31) == rk.RK_ERR_UNSUPPORTED
    assert call.dropout(back, rows=0) == rk.RK_OK


@pytest.mark.parametrize("way", ["loss", "backward", "both"])
def test_head_refuses(call, rk, way):
    m = call.matrix
    for bad in (dict(h=False), dict(scale=0.0), dict(scale=NAN), dict(scale=INF), dict(z=-1.0), dict(z=NAN), dict(z=INF), dict(width=0), dict(vocab=0), dict(width=65), dict(x=None),
                dict(weight=None), dict(x=m(type=rk.RK_F16)), dict(weight=m(type=rk.RK_F16)), dict(x=m(data=None)), dict(weight=m(data=0x1001)), dict(weight=m(stride=63)), dict(x=m(type=4)),
                dict(label=None), dict(label=0x1001), dict(row_weight=0x1002), dict(lse=None), dict(lse=0x1001)):
        assert call.head(way, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    for bad in [dict(loss=None), dict(total=None), dict(total=0x1002)] if way != "backward" else []:
        assert call.head(way, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    for bad in [dict(dx=None, d_weight=None), dict(dx=m(type=rk.RK_F32)), dict(d_weight=m(type=rk.RK_F16)), dict(dx=m(stride=63)), dict(d_weight=m(data=None)),
                dict(d_total=0x1001)] if way != "loss" else []:
        assert call.head(way, **bad) == rk.RK_ERR_INVALID_ARG and call.text(), bad
    wide = m(stride=70000)
    assert call.head(way, width=65537, x=wide, weight=wide) == rk.RK_ERR_UNSUPPORTED
    assert call.head(way, vocab=(1 << 28) + 1) == rk.RK_ERR_UNSUPPORTED
    assert call.head(way, rows=(1 << 20) + 1) == rk.RK_ERR_UNSUPPORTED


def test_the_binding_refuses_before_the_library(rk):
    import torch
    z = lambda *s, **k: torch.zeros(*s, **k)
    for bad in (dict(bias=z(2, 3)), dict(bias=z(8)[::2]), dict(offsets=z(3, dtype=torch.int32), seq_rows=4), dict(offsets=z(0, dtype=torch.int32)),
                dict(offsets=z(3, dtype=torch.int64)), dict(bias=z(4, dtype=torch.float64))):
        with pytest.raises(rk.RkError):
            rk.Recur(**bad)
    with pytest.raises(rk.RkError):
        rk.Dropout(0.5, z(2, dtype=torch.int32))
    with pytest.raises(rk.RkError):
        rk.Dropout(0.5, z(3, dtype=torch.int64))
    ctx = C.create_string_buffer(1 << 16)
    with pytest.raises(rk.RkError):                         # not on a GPU
        rk.rk_recur_forward(ctx, rk.Recur(), z(4, 8), z(4, 8), None, z(4, 8), None)
    with pytest.raises(rk.RkError):
        rk.rk_dropout_forward(ctx, rk.Dropout(0.5, z(2, dtype=torch.int64)), z(4, 8), None, z(4, 8))
    with pytest.raises(rk.RkError):
        rk.rk_head_loss(ctx, rk.make_head(), z(4, 8), z(9, 8), z(4, dtype=torch.int32), None, z(4), z(4), z(1))
    recur = rk.Recur(bias=z(8), seq_rows=3)
    assert recur._sizes(z(7, 8))[1] == (3, 8) and rk.Recur()._sizes(z(0, 5))[1] == (1, 5)
    assert rk.Recur(offsets=z(4, dtype=torch.int32))._sizes(z(7, 8))[1] == (3, 8)
    with pytest.raises(rk.RkError):
        recur._sizes(z(7, 9))
