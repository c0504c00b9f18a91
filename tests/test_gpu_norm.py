"""rk_norm_forward / rk_norm_backward against the plain form in 64 bits.

Tolerance of an element: half a step of its type (finfo.eps / 2, and half the smallest subnormal), and 2^-24 of the magnitudes that
enter it (oracle.training) times SUM: a row's sums are taken by lanes over at most 32 elements, then over 64 lanes and 16 wavefronts,
48 roundings at most, of two norms one after the other.  Sums over rows add a rounding a row.
"""
import numpy as np
import pytest

from oracle import training

pytestmark = pytest.mark.gpu
U32, SUM = 2.0 ** -24, 160.0
TINY = {"float16": 2.0 ** -25, "bfloat16": 2.0 ** -134, "float32": 2.0 ** -127}


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2408_08586_amd as rk
    ctx = rk.rk_create(0)
    yield torch, rk, ctx
    rk.rk_sync(ctx)
    rk.rk_destroy(ctx)


def close(torch, got, exact, size, what, terms=SUM, err=None):
    """err: what an input's own error adds."""
    g, e, s = got.double().cpu(), exact.double().cpu(), size.double().cpu()
    name = str(got.dtype)[6:]
    tol = (torch.finfo(got.dtype).eps / 2 if name != "float32" else 0.0) * e.abs() * (1 + 2.0 ** -8) + terms * U32 * s + TINY[name]
    bad = ~((g - e).abs() <= tol)
    same = (torch.isnan(g) & torch.isnan(e)) | (g == e)
    bad = bad & ~same
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} beyond the tolerance, the first at {bad.nonzero()[0].tolist()}: "
                                 f"{float(g[bad][0])!r} instead of {float(e[bad][0])!r} +- {float(tol[bad][0]):.2e}")


class Case:
    """Inputs of a block join on the GPU, made on the host from a seed."""

    def __init__(self, torch, rows, width, type="bfloat16", res=None, params=None, post="rms", pre="rms", vectors=("post_weight", "pre_weight"),
                 gate=None, gate_rows=0, pad=0, off=0, scale=1.0, seed=0, first=False, spread=1.0, shift=0.3):
        g = torch.Generator().manual_seed(seed * 7919 + rows * 31 + width)
        self.torch, self.rows, self.width, self.post, self.pre, self.scale = torch, rows, width, post, pre, scale
        self.t, self.r = getattr(torch, type), getattr(torch, res or type)
        self.p = getattr(torch, params or type)
        self.pad, self.off, self.gate_rows, self.first = pad, off, gate_rows, first
        n = lambda *s: torch.randn(*s, generator=g)
        self.x = self.rows_of(spread * n(rows, width) * (1 + n(width).abs()) + shift, self.r)
        self.y = None if first else self.rows_of(n(rows, width) * torch.exp(n(rows, 1)) + shift / 3, self.t)
        self.dxo = self.rows_of(0.1 * n(rows, width), self.r)
        self.du = self.rows_of(0.1 * n(rows, width), self.t)
        self.vec = {v: (n(width) * 0.3 + (1.0 if "weight" in v else 0.0)).to(self.p).cuda() for v in vectors}
        if gate is not None:
            self.vec["gate"] = (n(gate, width) * 0.5 + 0.5).to(self.p).cuda()
        self.double = {k: v.double().cpu() for k, v in self.vec.items()}

    def rows_of(self, values, dtype):
        """Rows `pad` elements apart, the first one `off` elements behind an aligned address."""
        torch = self.torch
        room = torch.full((self.rows * (self.width + self.pad) + self.off + 8,), float("nan"), dtype=dtype, device="cuda")
        m = room[self.off:self.off + self.rows * (self.width + self.pad)].view(self.rows, self.width + self.pad)[:, :self.width]
        if values is not None:
            m.copy_(values)
        return m

    def block(self, rk):
        return rk.NormBlock(post=self.post, pre=self.pre, res_scale=self.scale, gate_rows=self.gate_rows, **self.vec)

    def forward(self, rk, ctx):
        torch = self.torch
        x_out, u = self.rows_of(None, self.r), self.rows_of(None, self.t) if self.pre != "none" else None
        stats = torch.full((self.rows, 4), float("nan"), device="cuda")
        rk.rk_norm_forward(ctx, self.block(rk), self.x, self.y, x_out, u, stats)
        return x_out, u, stats

    def backward(self, rk, ctx, x_out, stats, dxo="given"):
        block = self.block(rk)
        grads = rk.NormGrads(block)
        for v in grads.tensors.values():
            v.fill_(float("nan"))
        dx, dy = self.rows_of(None, self.r), None if self.first else self.rows_of(None, self.t)
        du = self.du if self.pre != "none" else None
        dxo = self.dxo if dxo == "given" else None
        rk.rk_norm_backward(ctx, block, x_out, self.y, stats, dxo, du, dx, dy, grads if grads.tensors else None)
        return dx, dy, grads.tensors


def check(gpu, c, dxo="given"):
    torch, rk, ctx = gpu
    d = lambda t: None if t is None else t.double().cpu()
    x_out, u, stats = c.forward(rk, ctx)
    out, size = training.norm_forward(d(c.x), d(c.y), c.post, c.pre, c.double, c.gate_rows, c.scale, 1e-6, 1e-6)
    close(torch, x_out, out["x_out"], size["x_out"], "x_out")
    if u is not None:
        close(torch, u, out["u"], size["u"], "u", 2 * SUM)
    close(torch, stats, out["stats"], size["stats"] + out["stats"].abs(), "stats", 2 * SUM)
    dx, dy, grads = c.backward(rk, ctx, x_out, stats, dxo)
    out, size = training.norm_backward(d(x_out), d(c.y), d(stats), d(c.dxo) if dxo == "given" else None, d(c.du), c.post, c.pre, c.double,
                                       c.gate_rows, c.scale)
    close(torch, dx, out["dx"], size["dx"], "dx")
    if dy is not None:
        close(torch, dy, out["dy"], size["dy"], "dy", 2 * SUM)
    for name, v in grads.items():
        close(torch, v, out[name].reshape(v.shape), size[name].reshape(v.shape), "d_" + name, 2 * SUM + c.rows)


ALL = ("post_weight", "post_bias", "pre_weight", "pre_bias")


@pytest.mark.parametrize("rows,width", [(1, 1), (3, 2), (1, 7), (5, 64), (9, 129), (33, 512), (17, 513), (4, 1000), (7, 1025), (6, 2047), (3, 4099),
                                        (2, 8200), (2, 12288), (2, 16385), (1, 24704), (1, 32768)])
@pytest.mark.parametrize("type,res", [("bfloat16", None), ("float16", "float32"), ("float32", None)])
def test_widths(gpu, rows, width, type, res):
    check(gpu, Case(gpu[0], rows, width, type, res))


@pytest.mark.parametrize("type,res,params", [("float32", None, None), ("bfloat16", None, None), ("bfloat16", "float32", None), ("bfloat16", None, "float32"),
                                             ("bfloat16", "float32", "float32"), ("float16", None, "float32"), ("float16", "float32", None)])
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), ("none", "layer"), ("rms", "none"), ("layer", "rms")])
def test_types_and_kinds(gpu, type, res, params, post, pre):
    vectors = [v for v in ALL if not (post == "none" and "post" in v) and not (pre == "none" and "pre" in v)]
    check(gpu, Case(gpu[0], 21, 328, type, res, params, post, pre, vectors, gate=1, scale=0.75))
    check(gpu, Case(gpu[0], 13, 1500, type, res, params, post, pre, (), seed=1))


@pytest.mark.parametrize("rows,gate_rows", [(24, 1), (25, 2), (40, 5), (41, 7), (60, 8), (100, 33), (64, 64), (63, 100), (1, 1), (700, 300), (5000, 3)])
@pytest.mark.parametrize("width", [40, 2056])
def test_gates_of_rows(gpu, rows, gate_rows, width):
    check(gpu, Case(gpu[0], rows, width, gate=(rows + gate_rows - 1) // gate_rows, gate_rows=gate_rows, vectors=ALL, seed=2))


@pytest.mark.parametrize("pad,off", [(1, 0), (0, 1), (3, 3), (8, 0), (5, 2)])
@pytest.mark.parametrize("width", [61, 2048, 5003])
@pytest.mark.parametrize("type", ["bfloat16", "float32"])
def test_strides_and_alignments(gpu, pad, off, width, type):
    c = Case(gpu[0], 6, width, type, gate=1, pad=pad, off=off, vectors=ALL, post="layer", pre="layer")
    check(gpu, c)
    # nothing is written between the rows
    x_out, u, _ = c.forward(gpu[1], gpu[2])
    if pad:
        for t in (x_out, u):
            gap = t.as_strided((t.shape[0] - 1, pad), (t.stride(0), 1), t.storage_offset() + width)
            assert bool(gpu[0].isnan(gap).all())


@pytest.mark.parametrize("rows", [511, 1030, 4097, 9000])
def test_many_rows(gpu, rows):
    check(gpu, Case(gpu[0], rows, 136, gate=1, vectors=ALL))


def test_first_and_last_norm_of_a_stream(gpu):
    torch, rk, ctx = gpu
    c = Case(torch, 12, 384, post="none", first=True, vectors=("pre_weight",))
    check(gpu, c)
    check(gpu, c, dxo=None)
    # x_out not kept
    u, stats = c.rows_of(None, c.t), torch.empty(12, 4, device="cuda")
    rk.rk_norm_forward(ctx, c.block(rk), c.x, None, None, u, stats)
    assert torch.equal(u, c.forward(rk, ctx)[1])


def test_in_place(gpu):
    torch, rk, ctx = gpu
    c = Case(torch, 37, 2176, gate=1)
    x_out, u, stats = c.forward(rk, ctx)
    again = torch.empty_like(stats)
    rk.rk_norm_forward(ctx, c.block(rk), c.x, c.y, c.x, c.y, again)
    assert torch.equal(c.x, x_out) and torch.equal(c.y, u) and torch.equal(again, stats)


def test_means_far_from_zero(gpu):
    """A layer norm of rows whose mean is 4,096 times their spread: the squares about the mean do not cancel."""
    check(gpu, Case(gpu[0], 8, 5000, "float32", post="layer", pre="layer", spread=0.25, shift=3000.0, vectors=ALL))


def test_rows_that_are_not_finite_stay_alone(gpu):
    torch, rk, ctx = gpu
    c = Case(torch, 9, 640, post="layer", pre="layer", gate=1)
    clean = [t.clone() for t in c.forward(rk, ctx)]
    c.y[3, 17], c.x[6, 5] = float("nan"), float("inf")
    got = c.forward(rk, ctx)
    for a, b in zip(clean, got):
        rest = [r for r in range(9) if r not in (3, 6)]
        assert torch.equal(a[rest], b[rest])
    assert bool(torch.isnan(got[1][3]).all()) and not bool(torch.isfinite(got[1][6]).all())


def test_zero_rows_of_values(gpu):
    """A row of zeros: only eps is left under the root."""
    torch, rk, ctx = gpu
    c = Case(torch, 4, 96, "float32", post="rms", pre="layer", vectors=ALL)
    c.x.zero_(), c.y.zero_()
    check(gpu, c)


def test_no_rows(gpu):
    torch, rk, ctx = gpu
    c = Case(torch, 0, 300, gate=1, vectors=ALL)
    x_out, u, stats = c.forward(rk, ctx)
    _, _, grads = c.backward(rk, ctx, x_out, stats)
    for v in grads.values():
        assert bool((v == 0).all())


def test_gradient_against_differences(gpu):
    """Central differences of sum(a x_out + b u) in 64 bits along random directions, at float32 inputs."""
    torch, rk, ctx = gpu
    c = Case(torch, 5, 200, "float32", post="layer", pre="rms", gate=3, gate_rows=2, vectors=ALL, scale=0.9)
    x_out, u, stats = c.forward(rk, ctx)
    dx, dy, grads = c.backward(rk, ctx, x_out, stats)
    x, y, a, b = (t.double().cpu() for t in (c.x, c.y, c.dxo, c.du))

    def value(x, y, vec):
        out, _ = training.norm_forward(x, y, c.post, c.pre, vec, c.gate_rows, c.scale, 1e-6, 1e-6)
        return float((a * out["x_out"]).sum() + (b * out["u"]).sum())

    g = torch.Generator().manual_seed(5)
    for name, grad in [("x", dx), ("y", dy)] + list(grads.items()):
        way = torch.randn(grad.shape, generator=g, dtype=torch.float64)
        h, ends = 1e-5, []
        for s in (h, -h):
            vec = dict(c.double)
            if name in vec:
                vec[name] = vec[name] + s * way
            ends.append(value(x + s * way if name == "x" else x, y + s * way if name == "y" else y, vec))
        slope, formula = (ends[0] - ends[1]) / (2 * h), float((grad.double().cpu() * way).sum())
        size = float((grad.double().cpu() * way).abs().sum())
        assert abs(slope - formula) <= 2e-5 * size + 1e-6, (name, slope, formula)


def test_equal_calls_return_equal_bits_and_a_graph_replays_them(gpu):
    torch, rk, _ = gpu
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rk.rk_create(0)
        c = Case(torch, 300, 2176, gate=3, gate_rows=128, vectors=ALL)
        block = c.block(rk)
        grads = rk.NormGrads(block)
        x_out, u, dx, dy = (c.rows_of(None, c.t) for _ in range(4))
        stats = torch.empty(300, 4, device="cuda")

        def step():
            rk.rk_norm_forward(ctx, block, c.x, c.y, x_out, u, stats)
            rk.rk_norm_backward(ctx, block, x_out, c.y, stats, c.dxo, c.du, dx, dy, grads)

        everything = lambda: [t.clone() for t in (x_out, u, stats, dx, dy, *grads.tensors.values())]
        step()
        first = everything()
        step()
        for a, b in zip(first, everything()):
            assert torch.equal(a, b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for turn in range(3):
            c.x.mul_(1.25)
            graph.replay()
            replayed = everything()
            step()
            for a, b in zip(replayed, everything()):
                assert torch.equal(a, b), turn
        rk.rk_sync(ctx)
        rk.rk_destroy(ctx)
