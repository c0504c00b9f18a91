"""The training-step operators where their rules change path: by rows, widths, types and how gates, groups and slices fall.

Comparison and tolerances are those of the operators' own tests.
"""
import pytest

from oracle import training
from test_gpu_distill import Student
from test_gpu_norm import ALL, Case, check
from test_gpu_route import Route, logits_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2408_08586_amd as rk
    ctx = rk.rk_create(0)
    yield torch, rk, ctx
    rk.rk_sync(ctx)
    rk.rk_destroy(ctx)


# rows that a wavefront holds and ones that workgroups share; one and two vectors a lane; sums in registers and as a second pass
@pytest.mark.parametrize("width", [8, 500, 505, 512, 600, 767, 1024, 1029, 4096, 8192, 8200, 8576, 9999, 12288, 12296, 16384])
@pytest.mark.parametrize("type,res", [("bfloat16", None), ("float16", "float32"), ("float32", None)])
@pytest.mark.parametrize("vectors", [("post_weight", "pre_weight"), ALL])
def test_norm_widths_with_few_rows(gpu, width, type, res, vectors):
    check(gpu, Case(gpu[0], 7, width, type, res, gate=1, vectors=vectors, post="layer" if len(vectors) > 2 else "rms"))


@pytest.mark.parametrize("rows", [9, 255, 257, 300, 600, 2100])
@pytest.mark.parametrize("width,type", [(72, "bfloat16"), (999, "bfloat16"), (300, "float32"), (777, "float32"), (1300, "float16")])
def test_norm_rows(gpu, rows, width, type):
    check(gpu, Case(gpu[0], rows, width, type, gate=1, vectors=ALL, post="layer", pre="layer"))
    check(gpu, Case(gpu[0], rows, width, type, gate=(rows + 99) // 100, gate_rows=100, vectors=ALL, seed=1))


@pytest.mark.parametrize("width", [250, 8600])
@pytest.mark.parametrize("rows,gate_rows", [(530, 1), (530, 2), (530, 3), (530, 7), (530, 64), (530, 263), (530, 529), (40, 39)])
def test_norm_gates_by_chunk(gpu, width, rows, gate_rows):
    if width > 1000:
        rows, gate_rows = min(rows, 90), min(gate_rows, 44)
    check(gpu, Case(gpu[0], rows, width, gate=(rows + gate_rows - 1) // gate_rows, gate_rows=gate_rows, vectors=ALL, seed=4))


@pytest.mark.parametrize("width", [300, 2200, 9000, 13000])
def test_norm_gradients_that_are_not_asked_for(gpu, width):
    """Any part of the vectors' gradients, or none, leaves the others and the rows' as they are."""
    torch, rk, ctx = gpu
    c = Case(torch, 30, width, gate=3, gate_rows=10, vectors=ALL)
    x_out, u, stats = c.forward(rk, ctx)
    dx, dy, grads = c.backward(rk, ctx, x_out, stats)
    block = c.block(rk)
    for names in ((), ("gate",), ("pre_bias",), ("post_weight", "pre_weight"), ("post_bias", "gate")):
        some = rk.NormGrads(block, names)
        ex, ey = c.rows_of(None, c.r), c.rows_of(None, c.t)
        rk.rk_norm_backward(ctx, block, x_out, c.y, stats, c.dxo, c.du, ex, ey, some if names else None)
        # (without any of the sums the rows take another kernel, whose sums run in another order)
        tol = dict(rtol=2 ** -7, atol=1e-3) if not names else dict(rtol=0, atol=0)
        torch.testing.assert_close(ex, dx, **tol)
        torch.testing.assert_close(ey, dy, **tol)
        # (how many vectors there are decides how a sum's 30 rows are shared out: 64 roundings of sums of sizes below 120)
        for n, t in some.tensors.items():
            torch.testing.assert_close(t, grads[n], rtol=0, atol=64 * 2 ** -24 * 120)


def test_norm_rows_far_apart(gpu):
    """Rows more than 2^31 elements from each other."""
    torch, rk, ctx = gpu
    far = (1 << 31) + 40
    room = {n: torch.empty(2 * far + 512, dtype=torch.bfloat16, device="cuda") for n in ("a", "b")}
    at = lambda n, o: room[n].as_strided((3, 512), (far, 1), o)
    c = Case(torch, 3, 512, gate=1)
    x, y, xo, u = at("a", 0).copy_(c.x), at("b", 0).copy_(c.y), at("a", 0), at("b", 0)
    want = c.forward(rk, ctx)
    stats = torch.empty(3, 4, device="cuda")
    rk.rk_norm_forward(ctx, c.block(rk), x, y, xo, u, stats)
    for a, b in zip((xo, u, stats), want):
        assert torch.equal(a, b)


def test_norm_graph_of_a_wide_block(gpu):
    """Kernels with more LDS than a launch has by itself, in a graph."""
    torch, rk, _ = gpu
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rk.rk_create(0)
        c = Case(torch, 40, 8576, gate=1, vectors=ALL)
        s = Student((torch, rk, ctx), 300, 40000, 8, "bfloat16", kd=0.5, ce=0.5)
        r = Route((torch, rk, ctx), logits_of(torch, 900, 700, "bfloat16"), None, 4, True, 300)
        block = c.block(rk)
        grads, stats = rk.NormGrads(block), torch.empty(40, 4, device="cuda")
        x_out, u, dx, dy = (c.rows_of(None, c.t) for _ in range(4))
        out, d = [torch.empty(n, device="cuda") for n in ((300,), (300, 2), (1,))], torch.empty_like(s.s)
        dl, dw, dr = torch.tensor([0.1, 0.2], device="cuda"), torch.randn(900, 4, device="cuda"), torch.empty_like(r.logits)
        o = r.out

        def step():
            rk.rk_norm_forward(ctx, block, c.x, c.y, x_out, u, stats)
            rk.rk_norm_backward(ctx, block, x_out, c.y, stats, c.dxo, c.du, dx, dy, grads)
            rk.rk_distill_loss_backward(*s.given(), s.d_total, *out, d)
            r.forward()
            rk.rk_route_backward(ctx, r.router, r.logits, o["expert"], o["lse"], o["counts"], o["tokens"], dl, dw, dr)

        everything = lambda: [t.clone() for t in (x_out, u, stats, dx, dy, *grads.tensors.values(), *out, d, *o.values(), dr)]
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for turn in range(3):
            for t in (c.x, s.s, r.logits):
                t.mul_(1.125)
            graph.replay()
            replayed = everything()
            step()
            for a, b in zip(replayed, everything()):
                assert torch.equal(a, b), turn
        rk.rk_sync(ctx)
        rk.rk_destroy(ctx)


# tokens of one workgroup, of several, of more rounds than one; groups shorter than a round
@pytest.mark.parametrize("n,e,group", [(32, 160, 0), (128, 160, 0), (129, 160, 0), (256, 64, 0), (257, 64, 0), (700, 33, 20), (66000, 8, 0), (70000, 12, 9000), (400, 1000, 130)])
@pytest.mark.parametrize("dtype", ["float32", "float16"])
def test_route_by_tokens(gpu, n, e, group, dtype):
    Route(gpu, logits_of(gpu[0], n, e, dtype), None, min(3, e), True, group).check()


@pytest.mark.parametrize("e", [8, 32, 33, 64, 66, 128, 131, 192, 196, 256, 512, 600, 1024])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("k", [1, 8, 17, 32])
def test_route_experts_and_choices(gpu, e, dtype, k):
    torch = gpu[0]
    l = logits_of(torch, 90, e, dtype)
    l[3] = torch.finfo(l.dtype).max
    l[4, ::3] = float("-inf")
    l[5] = (torch.arange(e) % 5).to(l.dtype)
    l[6] = -(torch.arange(e) % 7).to(l.dtype) * torch.finfo(l.dtype).tiny     # the smallest numbers that are normal
    l[3] = l[3] * 0                                                            # (as lse: a row of zeros)
    Route(gpu, l, torch.arange(90) % 9 != 8, min(k, e), bool(k & 1), 40, pad=1).check()


def test_route_refuses_foreign_choices(gpu):
    """Choices outside the experts (as of another router) are none: nothing is read or written there."""
    torch, rk, ctx = gpu
    r = Route(gpu, logits_of(torch, 50, 24, "bfloat16"), None, 4)
    o = r.forward()
    d_loss, dw = torch.tensor([0.1, 0.2], device="cuda"), torch.randn(50, 4, device="cuda")
    d = r.backward(d_loss, dw)
    o["expert"][7] = torch.tensor([2 ** 30, -5, 24, 1000], dtype=torch.int32)
    e = r.backward(d_loss, dw)
    rest = [t for t in range(50) if t != 7]
    assert torch.equal(d[rest], e[rest]) and bool((e[7] == 0).all())


# vocabularies in one, four and eight vectors a thread, in LDS, and beyond; rows whole and in slices
@pytest.mark.parametrize("rows,vocab,dtype,k", [(260, 4096, "bfloat16", 256), (260, 4097, "bfloat16", 257), (260, 4099, "float16", 9), (260, 16384, "bfloat16", 30), (260, 16389, "bfloat16", 30),
                                                (260, 2048, "float32", 16), (260, 8195, "float32", 12), (260, 32776, "bfloat16", 700), (260, 20001, "float32", 40), (1030, 4096, "bfloat16", 256),
                                                (1030, 4097, "bfloat16", 257), (1030, 2048, "float32", 16), (1030, 8195, "float32", 12)])
def test_distill_by_vocabulary(gpu, rows, vocab, dtype, k):
    Student(gpu, rows, vocab, k, dtype, kd=0.5, ce=0.5, tau=1.0 if vocab % 2 else 2.0).check()


@pytest.mark.parametrize("vocab,dtype", [(66000, "bfloat16"), (140007, "bfloat16"), (70001, "float32"), (150000, "float16")])
def test_distill_rows_longer_than_what_is_kept(gpu, vocab, dtype):
    Student(gpu, 256, vocab, 20, dtype, kd=0.5, ce=0.5, tau=3.5, weights=False).check()


@pytest.mark.parametrize("rows,vocab", [(5, 900), (3, 90000), (260, 900), (256, 70000)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("tau", [1.0, 2.0, 3.0])
def test_distill_rows_masked_by_the_lowest_value(gpu, rows, vocab, dtype, tau):
    """Every word masked by the type's lowest value: an even distribution, not an overflow.  A row of them among others."""
    torch = gpu[0]
    s = Student(gpu, rows, vocab, 6, dtype, kd=0.5, ce=0.5, tau=tau, weights=False)
    low = torch.finfo(s.s.dtype).min
    s.s[1] = low
    s.s[2, vocab // 3:] = low
    s.ti[2] = torch.arange(6, dtype=torch.int32)
    s.label[2] = 4
    out, d1, both, d2 = s.run()
    ref = s.reference()
    # the masked row: T x lse and every logit are low; what is left is log V, below low's own steps, so its loss is not looked at
    rest = [r for r in range(rows) if r != 1]
    for o in (out, both):
        torch.testing.assert_close(o["loss"][rest].double().cpu(), ref["loss"][rest], rtol=2e-5, atol=2e-5)
        assert bool(torch.isfinite(o["lse"]).all()) and not bool(torch.isnan(o["loss"]).any())
    torch.testing.assert_close(d1[rest].double().cpu(), ref["d_student"][rest], rtol=2 ** -7, atol=1e-6)
    torch.testing.assert_close(d2[rest].double().cpu(), ref["d_student"][rest], rtol=2 ** -7, atol=1e-6)
    assert bool(torch.isfinite(d1.float()).all()) and bool(torch.isfinite(d2.float()).all())


def test_distill_rows_far_apart(gpu):
    torch, rk, ctx = gpu
    far = (1 << 31) + 8
    s = Student(gpu, 3, 3000, 5, "bfloat16", kd=0.5, ce=0.5)
    _, d1, both, d2 = s.run()
    room = torch.empty(2 * far + 3000, dtype=torch.bfloat16, device="cuda").as_strided((3, 3000), (far, 1), 0)
    s.s = room.copy_(s.s)
    out = [torch.empty_like(t) for t in both.values()]
    rk.rk_distill_loss_backward(*s.given(), s.d_total, *out, s.s)
    assert torch.equal(s.s, d2)
    for a, b in zip(out, both.values()):
        assert torch.equal(a, b)


def test_contexts_on_streams_of_their_own(gpu):
    """Two contexts work on two streams at once, each with its own buffers."""
    torch, rk, _ = gpu
    jobs = []
    for i in range(2):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            ctx = rk.rk_create(0)
            c, r = Case(torch, 200, 1400, gate=1, vectors=ALL, seed=i), Route((torch, rk, ctx), logits_of(torch, 3000, 64, seed=i), None, 4, True, 500)
            x_out, u, stats = c.forward(rk, ctx)
            want = [t.clone() for t in (*c.backward(rk, ctx, x_out, stats)[2].values(), *r.forward().values())]
            jobs.append((stream, ctx, c, r, x_out, stats, want))
    torch.cuda.synchronize()
    got = []
    for turn in range(5):
        for stream, ctx, c, r, x_out, stats, want in jobs:
            with torch.cuda.stream(stream):
                got.append((want, [t.clone() for t in (*c.backward(rk, ctx, x_out, stats)[2].values(), *r.forward().values())]))
    torch.cuda.synchronize()
    for want, have in got:
        for a, b in zip(want, have):
            assert torch.equal(a, b)
    for job in jobs:
        rk.rk_destroy(job[1])
