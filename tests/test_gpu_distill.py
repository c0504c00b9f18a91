"""rk_distill_loss / rk_distill_backward / rk_distill_loss_backward against the definition in 64 bits.

A softmax's sum over V elements is taken in lanes' runs of V / 64 at most (a row in one wavefront is the longest) and joined by up
to 64 more additions; each exponential is off by a few roundings of its argument.  So a row's sum, and whatever is divided by it, is off by
(V / 64 + TERMS) 2^-24 relatively, arguments by 2^-24 of the magnitudes that oracle.training adds up.
"""
import pytest

from oracle import training

pytestmark = pytest.mark.gpu
U32, TERMS = 2.0 ** -24, 96.0


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2408_08586_amd as rk
    ctx = rk.rk_create(0)
    yield torch, rk, ctx
    rk.rk_sync(ctx)
    rk.rk_destroy(ctx)


class Student:
    def __init__(self, gpu, rows, vocab, k=8, dtype="float32", teacher=None, tau=1.0, kd=1.0, ce=0.0, pad=0, off=0, weights=True, seed=0, spread=3.0):
        torch, self.rk, self.ctx = gpu
        self.torch, self.rows, self.vocab, self.tau, self.kd, self.ce = torch, rows, vocab, tau, kd, ce
        g = torch.Generator().manual_seed(seed * 977 + rows * 13 + vocab)
        t = getattr(torch, dtype)
        room = torch.full((rows * (vocab + pad) + off + 8,), float("nan"), dtype=t, device="cuda")
        self.s = room[off:off + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
        self.s.copy_(spread * torch.randn(rows, vocab, generator=g))
        k = min(k, vocab)
        self.tl = (spread * torch.randn(rows, k, generator=g)).to(getattr(torch, teacher or dtype)).cuda() if kd else None
        self.ti = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(rows)]).to(torch.int32).cuda() if kd and rows else \
            (torch.zeros(0, k, dtype=torch.int32, device="cuda") if kd else None)
        self.label = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32).cuda() if ce else None
        self.w = (torch.rand(rows, generator=g) * 2 * (torch.rand(rows, generator=g) > 0.2)).cuda() if weights else None
        self.d_total = torch.tensor([0.75], device="cuda")
        self.distill = self.rk.make_distill(tau, kd, ce)

    def given(self):
        return (self.ctx, self.distill, self.s, self.tl, self.ti, self.label, self.w)

    def run(self):
        torch = self.torch
        f = lambda *s: torch.full(s, float("nan"), device="cuda")
        out = dict(loss=f(self.rows), lse=f(self.rows, 2), total=f(1))
        self.rk.rk_distill_loss(*self.given(), *out.values())
        d1, d2 = torch.full_like(self.s, float("nan")), torch.full_like(self.s, float("nan"))
        self.rk.rk_distill_backward(*self.given(), out["lse"], self.d_total, d1)
        both = dict(loss=f(self.rows), lse=f(self.rows, 2), total=f(1))
        self.rk.rk_distill_loss_backward(*self.given(), self.d_total, *both.values(), d2)
        return out, d1, both, d2

    def reference(self):
        h = lambda t: None if t is None else t.cpu()
        d = lambda t: None if t is None else t.double().cpu()
        return training.distill(d(self.s), d(self.tl), h(self.ti), h(self.label), d(self.w), self.tau, self.kd, self.ce, 0.75)

    def check(self):
        torch = self.torch
        ref = self.reference()
        out, d1, both, d2 = self.run()
        terms = TERMS + self.vocab / 64
        s = self.s.double().cpu()
        top = s.masked_fill(~torch.isfinite(s), 0.0).abs().max(1).values if self.rows else s.new_zeros(0)
        for got in (out, both):
            self.near(got["lse"], ref["lse"], U32 * (terms + 8 * (top[:, None] / min(1.0, self.tau) + ref["lse"].abs().nan_to_num(posinf=0.0))), "lse")
            tol = terms * U32 * (ref["big_loss"] + ref["loss"].abs() + self.kd * self.tau ** 2 + self.ce)
            self.near(got["loss"], ref["loss"], tol, "loss")
            w = torch.ones(self.rows, dtype=torch.float64) if self.w is None else self.w.double().cpu()
            self.near(got["total"], ref["total"], (w * tol).sum().reshape(1) + 2 * U32 * ref["total"].abs(), "total")
        step = torch.finfo(self.s.dtype).eps / 2 if self.s.dtype != torch.float32 else 0.0
        tiny = 2.0 ** -25 if self.s.dtype == torch.float16 else 1e-37
        for d in (d1, d2):
            self.near(d, ref["d_student"], step * (1 + 2.0 ** -8) * ref["d_student"].abs() + terms * U32 * ref["big"] + tiny, "d_student")
        return ref, out, d1

    def near(self, got, want, tol, what):
        got = got.double().cpu()
        same = (got == want) | (self.torch.isnan(got) & self.torch.isnan(want))
        bad = ~((got - want).abs() <= tol) & ~same
        assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} beyond the tolerance at {bad.nonzero()[0].tolist()}: "
                                     f"{float(got[bad][0])!r} instead of {float(want[bad][0])!r}")


@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (3, 2, 2), (2, 7, 3), (5, 100, 8), (4, 1000, 64), (3, 4097, 33), (2, 32000, 100), (7, 8191, 256), (1, 50021, 64),
                                          (1, 128000, 1024), (40, 513, 5), (300, 260, 4), (1, 400003, 20)])
@pytest.mark.parametrize("kd,ce,tau", [(1.0, 0.0, 1.0), (0.6, 0.4, 2.0), (0.0, 1.0, 1.0)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_sizes(gpu, rows, vocab, k, kd, ce, tau, dtype):
    Student(gpu, rows, vocab, k, dtype, tau=tau, kd=kd, ce=ce).check()


@pytest.mark.parametrize("dtype,teacher", [("float32", "bfloat16"), ("bfloat16", "float32"), ("bfloat16", "float16"), ("float16", None), ("float16", "float32")])
@pytest.mark.parametrize("tau", [0.5, 1.0, 3.5])
@pytest.mark.parametrize("kd,ce", [(1.0, 0.0), (0.5, 0.5)])
def test_types_and_temperatures(gpu, dtype, teacher, tau, kd, ce):
    Student(gpu, 6, 3001, 50, dtype, teacher, tau, kd, ce).check()
    Student(gpu, 6, 3001, 50, dtype, teacher, tau, kd, ce, weights=False, seed=1).check()


@pytest.mark.parametrize("pad,off", [(1, 0), (0, 1), (3, 5), (8, 0)])
@pytest.mark.parametrize("vocab", [77, 5000, 40003])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides_and_alignments(gpu, pad, off, vocab, dtype):
    torch = gpu[0]
    s = Student(gpu, 4, vocab, 16, dtype, pad=pad, off=off, kd=0.5, ce=0.5, tau=2.0)
    s.check()
    wide = torch.full((4, vocab + pad + 4), 7.0, dtype=s.s.dtype, device="cuda")
    s.rk.rk_distill_loss_backward(*s.given(), s.d_total, *(torch.empty(n, device="cuda") for n in ((4,), (4, 2), (1,))), wide[:, 1:1 + vocab])
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, 1 + vocab:] == 7).all())


@pytest.mark.parametrize("rows", [255, 256, 257, 700, 1025])
@pytest.mark.parametrize("vocab", [600, 9001])
def test_many_rows(gpu, rows, vocab):
    Student(gpu, rows, vocab, 6, "bfloat16", kd=0.5, ce=0.5).check()


def test_indices_labels_and_teachers_that_are_not_there(gpu):
    torch = gpu[0]
    for dtype in ("float32", "bfloat16"):
        s = Student(gpu, 10, 1200, 6, dtype, kd=0.7, ce=0.3, tau=2.0, weights=False)
        inf = float("inf")
        s.ti[0, 2:] = -1
        s.ti[1] = -1                                     # no kept logit at all
        s.ti[2, 0], s.ti[2, 3] = 1200, 2 ** 31 - 1       # outside the vocabulary
        s.tl[3, 1] = -inf
        s.tl[4] = -inf                                   # none above -inf
        s.ti[5] = 77                                     # one index over and over
        s.ti[6, 1], s.ti[6, 4] = s.ti[6, 0], s.ti[6, 3]
        s.label[6] = s.ti[6, 0]                          # label among the teacher's
        s.label[7], s.label[8], s.label[1] = -100, 1200, -1
        s.tl[9, 0] = 80.0                                # one of them has everything: the others' q is zero
        s.check()


def test_rows_without_weight_are_not_looked_at(gpu):
    torch = gpu[0]
    s = Student(gpu, 6, 900, 5, "bfloat16", kd=0.5, ce=0.5)
    s.w[:] = 1.0
    s.w[2] = s.w[4] = 0.0
    s.s[2], s.s[4, 10], s.tl[2, 0] = float("nan"), float("inf"), float("nan")
    _, out, d = s.check()
    assert float(out["loss"][2]) == 0.0 and bool((d[2] == 0).all()) and bool(torch.isfinite(out["total"]).all())


def test_students_of_minus_infinity(gpu):
    """Masked words; a word that the teacher wants and the student excludes; nothing left at all; the type's lowest value as a mask."""
    torch, inf = gpu[0], float("inf")
    for dtype in ("float32", "bfloat16", "float16"):
        s = Student(gpu, 6, 700, 5, dtype, kd=0.5, ce=0.5, weights=False, tau=1.5)
        low = torch.finfo(s.s.dtype).min
        keep = s.ti[0].long()
        row = torch.full((700,), -inf, device="cuda", dtype=s.s.dtype)
        row[keep] = s.s[0, keep]
        s.label[0] = s.ti[0, 1]
        s.s[0] = row
        s.s[1] = -inf
        s.s[3, 350:] = low
        s.ti[3] = torch.arange(5, dtype=torch.int32)
        s.label[3] = 3
        ref, out, d = s.check()
        assert float(out["loss"][1]) == 0.0 and bool((d[1] == 0).all()) and float(out["lse"][1, 0]) == -inf
        s.s[2, int(s.ti[2, 0])] = -inf
        got, d1, _, _ = s.run()
        assert float(got["loss"][2]) == inf and bool(torch.isfinite(got["loss"][[0, 3, 4, 5]]).all()) and bool(torch.isfinite(d1.float()).all())


def test_rows_that_are_not_finite_stay_alone(gpu):
    torch = gpu[0]
    s = Student(gpu, 8, 2000, 5, "bfloat16", kd=0.5, ce=0.5, weights=False)
    clean, d, _, _ = s.run()
    s.s[2, 100], s.s[5, 7] = float("nan"), float("inf")
    got, e, _, f = s.run()
    rest = [0, 1, 3, 4, 6, 7]
    for k in ("loss", "lse"):
        assert torch.equal(clean[k][rest], got[k][rest])
    assert torch.equal(d[rest], e[rest]) and torch.equal(d[rest], f[rest])
    assert bool(torch.isnan(got["loss"][[2, 5]]).all()) and bool(torch.isnan(got["total"]).all()) and bool(torch.isnan(e[2].float()).all())


def test_large_logits(gpu):
    """Logits in the thousands: without the row's largest taken off first every exponential would overflow."""
    Student(gpu, 4, 3000, 6, "float32", spread=3000.0, kd=0.5, ce=0.5).check()


def test_no_rows(gpu):
    s = Student(gpu, 0, 500, 4, kd=0.5, ce=0.5)
    out, _, both, _ = s.run()
    assert float(out["total"]) == 0.0 and float(both["total"]) == 0.0


@pytest.mark.parametrize("rows", [3, 600])
def test_in_place(gpu, rows):
    torch = gpu[0]
    s = Student(gpu, rows, 7001, 20, "bfloat16", kd=0.5, ce=0.5, tau=2.0)
    _, d1, both, d2 = s.run()
    copy = s.s.clone()
    f = lambda *n: torch.empty(n, device="cuda")
    out = dict(loss=f(rows), lse=f(rows, 2), total=f(1))
    s.rk.rk_distill_loss_backward(*s.given(), s.d_total, *out.values(), s.s)
    assert torch.equal(s.s, d2)
    for k in out:
        assert torch.equal(out[k], both[k])
    s.s.copy_(copy)
    s.rk.rk_distill_backward(*s.given(), out["lse"], s.d_total, s.s)
    assert torch.equal(s.s, d1)


def test_gradient_against_differences(gpu):
    torch = gpu[0]
    s = Student(gpu, 4, 60, 7, "float32", tau=2.0, kd=0.6, ce=0.4, weights=False)
    grad = s.run()[1].double().cpu()
    x, way = s.s.double().cpu(), torch.randn(4, 60, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    ends = [float(training.distill(x + h * way, s.tl.double().cpu(), s.ti.cpu(), s.label.cpu(), None, 2.0, 0.6, 0.4)["total"]) for h in (1e-5, -1e-5)]
    slope, formula = 0.75 * (ends[0] - ends[1]) / 2e-5, float((grad * way).sum())
    assert abs(slope - formula) <= 2e-5 * float((grad * way).abs().sum()) + 1e-7


def test_equal_calls_return_equal_bits_and_a_graph_replays_them(gpu):
    torch, rk, _ = gpu
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rk.rk_create(0)
        for rows, vocab in ((5, 40000), (600, 3000)):
            s = Student((torch, rk, ctx), rows, vocab, 16, "bfloat16", kd=0.5, ce=0.5, tau=2.0)
            f = lambda *n: torch.empty(n, device="cuda")
            out, d = (f(rows), f(rows, 2), f(1)), torch.empty_like(s.s)
            d2, out2 = torch.empty_like(s.s), (f(rows), f(rows, 2), f(1))

            def step():
                rk.rk_distill_loss_backward(*s.given(), s.d_total, *out, d)
                rk.rk_distill_loss(*s.given(), *out2)
                rk.rk_distill_backward(*s.given(), out2[1], s.d_total, d2)

            everything = lambda: [t.clone() for t in (*out, *out2, d, d2)]
            step()
            first = everything()
            step()
            for a, b in zip(first, everything()):
                assert torch.equal(a, b)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                step()
            for turn in range(3):
                s.s.mul_(1.125)
                graph.replay()
                replayed = everything()
                step()
                for a, b in zip(replayed, everything()):
                    assert torch.equal(a, b), turn
        rk.rk_sync(ctx)
        rk.rk_destroy(ctx)
