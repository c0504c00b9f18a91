"""The training-step operators at the edges of what their header promises, each held against the definition in 64 bits or against a call
that needs no edge.  Tolerances are those of the operators' own tests, or derived where they are used.
"""
import pytest

from oracle import training
from test_gpu_distill import TERMS, U32, Student
from test_gpu_norm import ALL, Case
from test_gpu_route import Route, logits_of

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2408_08586_amd as rk
    ctx = rk.rk_create(0)
    yield torch, rk, ctx
    rk.rk_sync(ctx)
    rk.rk_destroy(ctx)


@pytest.mark.parametrize("rows,gate_rows,gates", [(15, 10, 5), (8, 10, 2), (10, 10, 3), (300, 7, 60), (3000, 2, 1600), (1, 1, 2), (0, 4, 3)])
@pytest.mark.parametrize("width", [40, 521, 2056, 13000])
def test_gates_without_rows_have_zero_gradients(gpu, rows, gate_rows, gates, width):
    """As in a shorter last batch: the gates behind the last row's are there, and no row uses them."""
    torch, rk, ctx = gpu
    if width > 3000 and rows > 300:
        rows, gates = 40, 33
    c = Case(torch, rows, width, gate=gates, gate_rows=gate_rows, vectors=ALL, seed=3)
    x_out, u, stats = c.forward(rk, ctx)
    dx, dy, grads = c.backward(rk, ctx, x_out, stats)
    used = (rows + gate_rows - 1) // gate_rows
    assert grads["gate"].shape[0] == gates and bool((grads["gate"][used:] == 0).all())
    c.vec["gate"] = c.vec["gate"][:max(used, 1)]
    ex, ey, exact = c.backward(rk, ctx, x_out, stats)
    assert torch.equal(dx, ex) and torch.equal(dy, ey)
    for name, v in exact.items():
        assert torch.equal(grads[name][:used] if name == "gate" else grads[name], v[:used] if name == "gate" else v), name
    # the gates' gradient alone, and in a call that follows one with more rows
    block = rk.NormBlock(post=c.post, pre=c.pre, gate_rows=gate_rows, **dict(c.vec, gate=torch.ones(gates, width, dtype=c.p, device="cuda")))
    alone = rk.NormGrads(block, ("gate",))
    alone.tensors["gate"].fill_(7.0)
    rk.rk_norm_backward(ctx, block, x_out, c.y, stats, c.dxo, c.du, dx, dy, alone)
    assert bool((alone.tensors["gate"][used:] == 0).all()) and bool(torch.isfinite(alone.tensors["gate"]).all())


def test_gates_without_rows_in_a_graph(gpu):
    torch, rk, _ = gpu
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rk.rk_create(0)
        c = Case(torch, 50, 300, gate=9, gate_rows=20, vectors=ALL)
        block = c.block(rk)
        grads = rk.NormGrads(block)
        x_out, u, stats = c.forward(rk, ctx)
        dx, dy = c.rows_of(None, c.r), c.rows_of(None, c.t)
        step = lambda: rk.rk_norm_backward(ctx, block, x_out, c.y, stats, c.dxo, c.du, dx, dy, grads)
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for turn in range(3):
            c.du.mul_(1.25)
            for v in grads.tensors.values():
                v.fill_(NAN)
            graph.replay()
            replayed = [t.clone() for t in (dx, dy, *grads.tensors.values())]
            step()
            for a, b in zip(replayed, (dx, dy, *grads.tensors.values())):
                assert torch.equal(a, b), turn
            assert bool((grads.tensors["gate"][3:] == 0).all())
        rk.rk_sync(ctx)
        rk.rk_destroy(ctx)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("n", [12, 1500])
def test_choices_that_are_not_there_have_weight_zero(gpu, dtype, renorm, n):
    """Also those of a token with a NaN, whose chosen ones have weight NaN."""
    torch = gpu[0]
    l = logits_of(torch, n, 48, dtype)
    l[1], l[2], l[3], l[4], l[5] = NAN, -INF, -INF, NAN, -INF
    l[2, 7] = NAN                                        # beside nothing but -inf
    l[3, 5], l[3, 9] = NAN, 1.0                          # two of them chosen
    l[3, 20] = 2.0
    l[4, 30] = 0.5                                       # one chosen
    l[6, 3] = NAN                                        # all chosen
    l[7] = -INF
    l[7, [4, 8]] = 1.0                                   # no NaN: two chosen, their weights as they are
    got = {k: v.cpu() for k, v in Route(gpu, l, None, 4, renorm).forward().items()}
    none = got["expert"] < 0
    assert none[[1, 2, 5]].all() and none[3].tolist() == none[7].tolist() == [False, False, True, True] and none[4].tolist() == [False, True, True, True]
    assert bool((got["weight"][none] == 0).all())
    assert bool(torch.isnan(got["weight"][[3, 4, 6]][~none[[3, 4, 6]]]).all()) \
        and bool(((got["weight"][7, :2] - 0.5).abs() <= 4 * U32).all())
    ref = training.route(l[:8].double(), None, 4, renorm, 0)
    assert torch.equal(ref["weight"].isnan(), got["weight"][:8].isnan()) and bool((ref["weight"][none[:8]] == 0).all())


@pytest.mark.parametrize("tau", [20.0, 100.0, 1e3, 1e5])
@pytest.mark.parametrize("rows,vocab", [(5, 1000), (5, 20001), (300, 1000)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_high_temperatures_leave_the_labels_loss_alone(gpu, tau, rows, vocab, dtype):
    """The label's probability is no less exact the higher the temperature of the other term, whether the gradient is taken by itself, of
    rows in slices or along with the loss.  (kd_weight 1 / T^2: both terms of the loss are of size one.)"""
    Student(gpu, rows, vocab, 8, dtype, tau=tau, kd=1 / tau ** 2, ce=0.5).check()


# steps of the type at the size: float16 2 and 16 and 32, bfloat16 2 and 512 and 2^23
@pytest.mark.parametrize("dtype,size,step", [("float16", -3000.0, 2.0), ("float16", 20000.0, 16.0), ("float16", -65504.0, 0.0), ("bfloat16", -300.0, 2.0),
                                             ("bfloat16", 1e5, 512.0), ("bfloat16", -1e9, 0.0), ("bfloat16", -1e28, 0.0), ("float32", -1e9, 0.0), ("float32", 70000.0, 0.25)])
@pytest.mark.parametrize("tau", [1.0, 2.0, 3.0])
@pytest.mark.parametrize("rows,vocab", [(4, 700), (260, 900), (4, 20001)])
def test_logits_far_from_zero(gpu, dtype, size, step, tau, rows, vocab):
    """Rows masked by a large value that is not the type's lowest, or shifted as a whole: loss and gradient in one call are those of the same
    logits less the row's largest.  A 16-bit student's exponents below 2^11 are rounded to 2^-14 twice, larger ones are taken from
    differences."""
    torch = gpu[0]
    s = Student(gpu, rows, vocab, 6, dtype, kd=0.5, ce=0.5, tau=tau, weights=False)
    g = torch.Generator().manual_seed(vocab)
    base = float(torch.tensor(size).to(s.s.dtype))
    near = step * torch.randint(-2, 3, (rows, vocab), generator=g)
    far = near.to(torch.float64) + base
    assert torch.equal(far.to(s.s.dtype).double(), far)
    s.s[1:4] = far[1:4].to(s.s.dtype).cuda()
    shifted = s.s.double().cpu()
    shifted = shifted - shifted.max(1, keepdim=True).values
    d = lambda t: t.double().cpu()
    ref = training.distill(shifted, d(s.tl), s.ti.cpu(), s.label.cpu(), None, tau, 0.5, 0.5, 0.75)
    _, d1, both, d2 = s.run()
    rounding = torch.finfo(s.s.dtype).eps / 2 if dtype != "float32" else 0.0
    tiny = 2.0 ** -25 if dtype == "float16" else 1e-37
    exponents = 2 * 2.0 ** -14 if dtype != "float32" else 0.0
    tol = rounding * (1 + 2.0 ** -8) * ref["d_student"].abs() + ((TERMS + vocab / 64) * U32 + exponents) * ref["big"] + tiny
    s.near(d2, ref["d_student"], tol, "d_student")
    # from the log sums, which are rounded to 32 bits: no probability beyond one
    most = (0.5 * tau + 0.5) * 0.75 * (1 + 2.0 ** -7)
    assert bool((d1.double().cpu().abs() <= most).all())
    assert bool(torch.isfinite(both["lse"]).all()) and bool(torch.isfinite(both["loss"]).all())


@pytest.mark.parametrize("rows,vocab", [(3, 40000), (700, 20000), (260, 70001)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_distill_in_place_by_slices(gpu, rows, vocab, dtype):
    """d_student may be student, also where several workgroups share a row and what the teacher wants lies in all of their parts."""
    torch = gpu[0]
    s = Student(gpu, rows, vocab, 200, dtype, kd=0.5, ce=0.5, tau=2.0)
    _, _, both, d2 = s.run()
    copy, d1 = s.s.clone(), torch.empty_like(s.s)
    s.rk.rk_distill_backward(*s.given(), both["lse"], s.d_total, d1)
    f = lambda *n: torch.empty(n, device="cuda")
    out = dict(loss=f(rows), lse=f(rows, 2), total=f(1))
    s.rk.rk_distill_loss_backward(*s.given(), s.d_total, *out.values(), s.s)
    assert torch.equal(s.s, d2)
    for k in out:
        assert torch.equal(out[k], both[k])
    s.s.copy_(copy)
    s.rk.rk_distill_backward(*s.given(), both["lse"], s.d_total, s.s)
    assert torch.equal(s.s, d1)


def test_more_norm_rows_than_one_launch_has(gpu):
    """A launch has fewer than 2^32 threads, 64 of them a row: rows beyond 2^26, of one element."""
    torch, rk, ctx = gpu
    rows = (1 << 26) + 70
    x = ((torch.arange(rows, device="cuda") % 251) - 125).to(torch.bfloat16)[:, None]
    y = ((torch.arange(rows, device="cuda") % 127) + 1).to(torch.bfloat16)[:, None]
    gate = torch.tensor([[0.5], [2.0]], dtype=torch.bfloat16, device="cuda")
    first = 1 << 25
    gate = torch.cat((gate, torch.tensor([[4.0]], dtype=torch.bfloat16, device="cuda")))
    block = rk.NormBlock(post="none", pre="none", gate=gate, gate_rows=first)
    x_out, stats = torch.full_like(x, NAN), torch.full((rows, 4), NAN, device="cuda")
    rk.rk_norm_forward(ctx, block, x, y, x_out, None, stats)
    g = gate.float()[torch.arange(rows, device="cuda") // first]
    assert torch.equal(x_out, (x.float() + g * y.float()).to(torch.bfloat16))
    assert bool((stats == torch.tensor([0.0, 1.0, 0.0, 1.0], device="cuda")).all())
    dx, dy = torch.full_like(x, NAN), torch.full_like(x, NAN)
    rk.rk_norm_backward(ctx, block, x_out, y, stats, x, None, dx, dy)
    assert torch.equal(dx, x) and torch.equal(dy, (g * x.float()).to(torch.bfloat16))


def test_more_distilled_rows_than_one_launch_has(gpu):
    """Rows of two words, 128 threads each: beyond 2^25 of them."""
    torch, rk, ctx = gpu
    rows = (1 << 25) + 70
    s = (torch.arange(2 * rows, device="cuda") % 13).float().view(rows, 2) / 4
    label = (torch.arange(rows, device="cuda") % 2).to(torch.int32)
    distill = rk.make_distill(kd_weight=0.0, ce_weight=1.0)
    w = torch.full((rows,), 1.0 / rows, device="cuda")
    f = lambda *n: torch.full(n, NAN, device="cuda")
    loss, lse, total, d = f(rows), f(rows, 2), f(1), f(rows, 2)
    # 2 x 2^-24 a term, of numbers up to 4
    x = s.double()
    want = torch.logsumexp(x, 1)
    right = x.gather(1, label.long()[:, None])[:, 0]
    p = torch.softmax(x, 1)
    p.scatter_add_(1, label.long()[:, None], torch.full_like(p[:, :1], -1.0))
    for both in (True, False):
        loss.fill_(NAN), d.fill_(NAN), total.fill_(NAN)
        if both:
            rk.rk_distill_loss_backward(ctx, distill, s, None, None, label, w, None, loss, lse, total, d)
        else:
            rk.rk_distill_loss(ctx, distill, s, None, None, label, w, loss, lse, total)
            rk.rk_distill_backward(ctx, distill, s, None, None, label, w, lse, None, d)
        assert bool(((lse[:, 1].double() - want).abs() <= 16 * U32 * 4).all())
        assert bool(((loss.double() - (want - right)).abs() <= 32 * U32 * 4).all())
        assert bool(((d.double() * rows - p).abs() <= 32 * U32).all())
        assert abs(float(total) - float((want - right).mean())) <= 64 * U32 * 4



@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("e,k", [(8, 4), (64, 6), (200, 8), (1024, 32)])
@pytest.mark.parametrize("n", [9, 1200])
def test_the_largest_finite_logits(gpu, dtype, e, k, n):
    """Tokens of the type's largest finite value, alone, beside its neighbour below and beside +inf: which are chosen, and in what order."""
    torch = gpu[0]
    l = logits_of(torch, n, e, dtype)
    top = torch.finfo(l.dtype).max
    below = torch.nextafter(torch.tensor(top, dtype=l.dtype), torch.tensor(0.0, dtype=l.dtype)) if dtype == "float32" else \
        torch.tensor([torch.tensor(top, dtype=l.dtype).view(torch.int16).item() - 1], dtype=torch.int16).view(l.dtype)[0]
    l[0] = top
    l[1] = below
    l[1, ::3] = top
    l[2, e // 2], l[2, e - 1] = top, top
    l[3] = -top
    l[3, 1::2] = top
    l[4] = top
    l[4, [1, e - 2]] = INF
    got = {name: v.cpu() for name, v in Route(gpu, l, None, k, True).forward().items()}
    for t in range(5):
        x = l[t].double()
        order = sorted(range(e), key=lambda i: (-float(x[i]), i))[:k]
        assert got["expert"][t].tolist() == order, t
    for t in range(4):                                   # (the fifth's softmax is not a number)
        x = l[t].double()
        w = torch.exp(x[got["expert"][t].long()] - x.max())
        assert float((got["weight"][t].double() - w / w.sum()).abs().max()) <= 64 * U32, t
        assert abs(float(got["lse"][t]) - float(torch.logsumexp(x, 0))) <= 2 * U32 * top
    assert bool(torch.isnan(got["lse"][4]))
