"""rk_head_loss / rk_head_backward / rk_head_loss_backward against the logits in 64 bits.

A logit is off by 2^-24 of the magnitudes of its products times their number over four and 32 (the matrix units add four products or more at
a time to a sum of 32 bits); lse by as much and a few units of its own; an element of the logits' gradient by that relative to its
probability, and by its rounding to the rows' type; sums over words and rows again by the number of their products over four and 32."""
import pytest

from oracle import training

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
TINY = {"float16": 2.0 ** -25, "bfloat16": 2.0 ** -134, "float32": 2.0 ** -126}


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2408_08586_amd as rk
    ctx = rk.rk_create(0)
    yield torch, rk, ctx
    rk.rk_sync(ctx)
    rk.rk_destroy(ctx)


def room(torch, rows, width, dtype, pad=0, off=0, values=None):
    stride = width + pad
    flat = torch.full((rows * stride + off + 8,), float("nan"), dtype=dtype, device="cuda")
    m = flat[off:off + rows * stride].view(rows, stride)[:, :width]
    return m if values is None else m.copy_(values)


class Case:
    def __init__(self, torch, rows, vocab, width, type="bfloat16", scale=1.0, z=0.0, weights=True, ignored=0.0, pad=0, off=0, d_total=1.0, seed=0, spread=2.0):
        g = torch.Generator().manual_seed(seed * 17 + rows + vocab + width)
        self.torch, self.t = torch, getattr(torch, type)
        self.shape, self.scale, self.z, self.pad, self.off = (rows, vocab, width), scale, z, pad, off
        n = lambda *s: torch.randn(*s, generator=g)
        self.x = self.matrix(rows, n(rows, width))
        self.weight = self.matrix(vocab, n(vocab, width) * (spread / (width ** 0.5 * abs(scale))))
        self.label = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
        gone = torch.rand(rows, generator=g) < ignored
        self.label[gone] = torch.tensor([-1, -100, vocab, 2 ** 31 - 1])[torch.randint(0, 4, (rows,), generator=g)][gone].to(torch.int32)
        self.label = self.label.cuda()
        self.row_weight = (0.5 + torch.rand(rows, generator=g)).cuda() if weights else None
        if weights and ignored:
            self.row_weight[::7] = 0.0
        self.d_total = torch.tensor([d_total], device="cuda")

    def matrix(self, rows, values=None):
        return room(self.torch, rows, self.shape[2], self.t, self.pad, self.off, values)

    def outputs(self):
        torch, (rows, vocab, width) = self.torch, self.shape
        f = lambda *s: torch.full(s, float("nan"), device="cuda")
        return {"loss": f(rows), "lse": f(rows), "total": f(1), "dx": self.matrix(rows), "d_weight": self.matrix(vocab)}

    def given(self, rk, ctx):
        return ctx, rk.make_head(logit_scale=self.scale, z_weight=self.z), self.x, self.weight, self.label, self.row_weight

    def run(self, rk, ctx):
        """Loss and gradients apart, and both at once."""
        one, two = self.outputs(), self.outputs()
        rk.rk_head_loss(*self.given(rk, ctx), one["loss"], one["lse"], one["total"])
        rk.rk_head_backward(*self.given(rk, ctx), one["lse"], self.d_total, one["dx"], one["d_weight"])
        rk.rk_head_loss_backward(*self.given(rk, ctx), self.d_total, two["loss"], two["lse"], two["total"], two["dx"], two["d_weight"])
        return one, two

    def check(self, rk, ctx):
        torch, (rows, vocab, width) = self.torch, self.shape
        c = lambda t: None if t is None else t.double().cpu()
        exact, size = training.head(c(self.x), c(self.weight), self.label.cpu(), c(self.row_weight), self.scale, self.z, c(self.d_total))
        name = str(self.t)[6:]
        half = torch.finfo(self.t).eps / 2 if name != "float32" else 0.0
        logit = (width / 4 + 32) * U32
        tol = {k: (logit * size[k] + 64 * U32 * (exact[k].abs() + 1)) for k in ("loss", "lse")}
        tol["total"] = (logit + (rows / 1024 + 64) * U32) * size["total"] + U32 * exact["total"].abs()
        most = float(size["big"].max()) if "big" in size else 0.0
        p = 2 * logit * most + 64 * U32                     # of a probability: its logit's and its row's lse's error
        steps = max(vocab, rows) / 4 + 64
        for k in ("dx", "d_weight"):
            # float16: the smallest numbers that are kept of a row are 2^-39 of its largest; of other types, probabilities below
            # 2^-126 are zero (an exponential has no smaller result): each adds up to 2^-126 times what it is multiplied by, one for every word
            # (dx) or row (d_weight)
            sums = (c(self.weight).abs().sum(0)[None] if k == "dx" else c(self.x).nan_to_num(0.0).abs().sum(0)[None])
            scale = float((c(self.row_weight).abs().max() if self.row_weight is not None else 1.0) if rows else 0.0) * abs(float(self.d_total)) * abs(self.scale)
            tol[k] = (half + p + steps * U32) * size[k] + half * exact[k].abs() * (1 + 2.0 ** -8) + TINY[name] + 2.0 ** (-39 if name == "float16" else -126) * 4 * scale * sums
        for which, out in zip(("apart", "at once"), self.run(rk, ctx)):
            for k, v in out.items():
                g, e = v.double().cpu(), exact[k]
                bad = ~((g - e).abs() <= tol[k])
                assert not bool(bad.any()), (f"{which} {k}: {int(bad.sum())} of {bad.numel()} beyond the tolerance, the first at {bad.nonzero()[0].tolist()}: "
                                             f"{float(g[bad][0])!r} instead of {float(e[bad][0])!r} +- {float(tol[k].expand_as(e)[bad][0]):.2e}")
            gone = exact["lse"] == 0
            assert bool((out["loss"].cpu()[gone] == 0).all()) and bool((out["dx"].cpu()[gone] == 0).all())


TYPES = ("bfloat16", "float16", "float32")


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("rows, vocab, width, pad, off", [(1, 1, 1, 0, 0), (1, 300, 64, 0, 0), (5, 1000, 128, 0, 0), (17, 257, 65, 0, 1), (40, 513, 200, 3, 0),
                                                            (64, 700, 72, 8, 8), (130, 999, 333, 1, 0), (300, 1500, 264, 0, 0), (513, 256, 48, 0, 0), (33, 5000, 40, 0, 0)])
def test_sizes(gpu, type, rows, vocab, width, pad, off):
    torch, rk, ctx = gpu
    Case(torch, rows, vocab, width, type, pad=pad, off=off, z=1e-3).check(rk, ctx)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("scale, z, ignored, d_total", [(0.5, 0.0, 0.3, 3.0), (-2.0, 0.01, 0.9, 1.0), (1.0, 2.0, 0.1, 0.125), (1.0, 0.0, 1.0, 1.0)])
def test_scales_and_rows_that_are_left_out(gpu, type, scale, z, ignored, d_total):
    torch, rk, ctx = gpu
    c = Case(torch, 150, 400, 96, type, scale=scale, z=z, ignored=ignored, d_total=d_total)
    # whatever they hold
    gone = (c.label < 0) | (c.label >= 400) | (c.row_weight == 0)
    keep = c.x.clone()
    one, _ = c.run(rk, ctx)
    c.x[gone] = float("nan")
    c.row_weight[c.label < 0] = float("nan")
    again, _ = c.run(rk, ctx)
    for k in one:
        assert torch.equal(one[k], again[k]), k
    c.x.copy_(keep)
    c.row_weight[c.label < 0] = 1.0
    c.check(rk, ctx)


def test_weights_of_very_different_rows(gpu):
    """A row's gradient has its own scale, whatever the other rows' weights; without weights all are ones."""
    torch, rk, ctx = gpu
    for type in TYPES:
        c = Case(torch, 60, 300, 64, type, weights=False)
        c.check(rk, ctx)
        c.row_weight = torch.logspace(-6, 3, 60).cuda()
        c.row_weight[::3] *= -1
        if type != "float16":
            c.check(rk, ctx)


def test_large_logits(gpu):
    """Logits in the hundreds: no exponential runs over."""
    torch, rk, ctx = gpu
    for type in ("bfloat16", "float32"):
        Case(torch, 20, 600, 128, type, spread=120.0).check(rk, ctx)


def test_one_gradient_alone(gpu):
    torch, rk, ctx = gpu
    c = Case(torch, 90, 700, 120, ignored=0.2)
    one, _ = c.run(rk, ctx)
    for want in ("dx", "d_weight"):
        out = c.outputs()
        rk.rk_head_backward(*c.given(rk, ctx), one["lse"], c.d_total, out["dx"] if want == "dx" else None, out["d_weight"] if want == "d_weight" else None)
        assert torch.equal(out[want], one[want])
        out = c.outputs()
        rk.rk_head_loss_backward(*c.given(rk, ctx), None, out["loss"], out["lse"], out["total"], out["dx"] if want == "dx" else None, out["d_weight"] if want == "d_weight" else None)
        assert torch.equal(out["loss"], one["loss"])


def test_no_rows(gpu):
    torch, rk, ctx = gpu
    c = Case(torch, 0, 100, 32, weights=False)
    for out in c.run(rk, ctx):
        assert float(out["total"]) == 0.0 and bool((out["d_weight"] == 0).all())


def test_nans_stay_in_their_rows(gpu):
    torch, rk, ctx = gpu
    c = Case(torch, 40, 500, 64, "float32")
    clean, _ = c.run(rk, ctx)
    c.x[7, 3] = float("nan")
    out, _ = c.run(rk, ctx)
    other = [r for r in range(40) if r != 7]
    assert bool(torch.isnan(out["loss"][7])) and bool(torch.isnan(out["dx"][7]).all()) and bool(torch.isnan(out["total"]).all())
    assert torch.equal(out["loss"][other], clean["loss"][other]) and torch.equal(out["dx"][other], clean["dx"][other])


def test_equal_calls_return_equal_bits_and_graphs(gpu):
    torch, rk, _ = gpu
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rk.rk_create(0)
        c = Case(torch, 300, 2000, 192, ignored=0.2)
        one, two = c.run(rk, ctx)
        again, _ = c.run(rk, ctx)
        assert all(torch.equal(one[k], again[k]) for k in one)
        out = c.outputs()

        def both():
            rk.rk_head_loss_backward(*c.given(rk, ctx), c.d_total, out["loss"], out["lse"], out["total"], out["dx"], out["d_weight"])

        both()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            both()
        for i in range(4):
            c.x.copy_(c.x.float() * 0.9 + 0.1)
            c.label.copy_(torch.roll(c.label, 1))
            both()
            want = {k: v.clone() for k, v in out.items()}
            for v in out.values():
                v.zero_()
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(out[k], want[k]) for k in out), i
        rk.rk_sync(ctx)
        rk.rk_destroy(ctx)


def test_gradients_are_differences(gpu):
    torch, rk, ctx = gpu
    c = Case(torch, 12, 90, 24, "float32", z=0.02, ignored=0.2)
    _, out = c.run(rk, ctx)
    g = torch.Generator().manual_seed(2)

    def total():
        f = lambda *s: torch.empty(*s, device="cuda")
        loss = f(12)
        rk.rk_head_loss(*c.given(rk, ctx), loss, f(12), f(1))
        return float((loss.double() * c.row_weight.double()).sum())

    for what, grad in ((c.x, out["dx"]), (c.weight, out["d_weight"])):
        way, keep, eps = torch.randn(what.shape, generator=g).cuda(), what.clone(), 2.0 ** -7
        what.copy_(keep + eps * way)
        up = total()
        what.copy_(keep - eps * way)
        down = total()
        what.copy_(keep)
        slope, want = (up - down) / (2 * eps), float((grad.double() * way.double()).sum())
        scale = float((grad.double() * way.double()).abs().sum())
        assert abs(slope - want) <= 100 * eps ** 2 * scale + 12 * 2.0 ** -21 / eps, (slope, want)


def test_several_pieces_of_the_vocabulary(gpu):
    """More gradients than the working buffer holds at once, labels in every piece; rows that need padding and rows that do not.  Against
    64 bits on the GPU, a norm of each result: 16-bit results are off by half a step each, the gradients' rounding by as much again."""
    torch, rk, ctx = gpu
    rows, vocab, half = 4200, 140001, torch.finfo(torch.bfloat16).eps / 2
    for width in (40, 33):
        g = torch.Generator("cuda").manual_seed(width)
        n = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
        x, words = n(rows, width), n(vocab, width) * 0.5
        label = torch.randint(0, vocab, (rows,), generator=g, device="cuda").int()
        label[:3] = torch.tensor([0, vocab - 1, -1])
        f = lambda *s: torch.full(s, float("nan"), device="cuda")
        loss, lse, total, dx, dw = f(rows), f(rows), f(1), n(rows, width), n(vocab, width)
        given = (ctx, rk.make_head(), x, words, label, None)
        rk.rk_head_loss_backward(*given, None, loss, lse, total, dx, dw)
        dx2, dw2 = torch.empty_like(dx), torch.empty_like(dw)
        rk.rk_head_backward(*given, lse, None, dx2, dw2)
        want_dw, want_dx, want_lse = torch.zeros(vocab, width, dtype=torch.float64, device="cuda"), [], []
        w64 = words.double()
        for a in range(0, rows, 700):
            x64 = x[a:a + 700].double()
            l = x64 @ w64.t()
            want_lse.append(torch.logsumexp(l, 1))
            p = torch.softmax(l, 1)
            keep = label[a:a + 700] >= 0
            p[torch.arange(len(p), device="cuda")[keep], label[a:a + 700][keep].long()] -= 1
            p[~keep] = 0
            want_dx.append(p @ w64)
            want_dw += p.t() @ x64
        want_dx, want_lse = torch.cat(want_dx), torch.cat(want_lse)
        assert float((lse.double() - want_lse)[3:].abs().max()) <= 64 * U32 * float(want_lse.max())
        for got, want in ((dx, want_dx), (dx2, want_dx), (dw, want_dw), (dw2, want_dw)):
            assert float((got.double() - want).norm()) <= 2 * half * float(want.norm())
            assert float((got.double() - want).abs().max()) <= 4 * half * float(want.abs().max())


def test_more_rows_than_the_sums_of_all_tiles_have_room_for(gpu):
    torch, rk, ctx = gpu
    rows, vocab, width = 1 << 18, 33001, 8
    g = torch.Generator("cuda").manual_seed(1)
    x, words = (torch.randn(n, width, generator=g, device="cuda").to(torch.bfloat16) for n in (rows, vocab))
    label = torch.randint(0, vocab, (rows,), generator=g, device="cuda").int()
    f = lambda *s: torch.full(s, float("nan"), device="cuda")
    loss, lse, total = f(rows), f(rows), f(1)
    rk.rk_head_loss(ctx, rk.make_head(), x, words, label, None, loss, lse, total)
    for a in (0, 100000, rows - 500):
        l = x[a:a + 500].double() @ words.double().t()
        want = torch.logsumexp(l, 1)
        assert float((lse[a:a + 500].double() - want).abs().max()) <= 64 * U32 * float(want.max())
        own = want - l[torch.arange(500, device="cuda"), label[a:a + 500].long()]
        assert float((loss[a:a + 500].double() - own).abs().max()) <= 128 * U32 * float(want.max())
    assert abs(float(total) - float(loss.double().sum())) <= U32 * float(total)


@pytest.mark.parametrize("type", ("bfloat16", "float16"))
@pytest.mark.parametrize("rows, vocab, width", [(4500, 600, 264), (2100, 40, 33), (33, 300, 520)])
def test_labels_that_meet_in_a_tile(gpu, type, rows, vocab, width):
    """What rounding takes off the labels' gradients is there, of however many rows have one label: what d_weight is off by are other words'
    roundings and its own, and of its labels' rows the rounding of a rounding."""
    torch, rk, ctx = gpu
    c = Case(torch, rows, vocab, width, type)
    words = torch.tensor([vocab - 1, 0, min(255, vocab - 1), min(256, vocab - 1)], dtype=torch.int32).cuda()
    few = torch.arange(rows, device="cuda") % 50 < 4
    c.label[~few] = 7
    c.label[few] = words[torch.arange(rows, device="cuda")[few] % 4]
    c.check(rk, ctx)
    x, w, label, weight = c.x.double().cpu(), c.weight.double().cpu(), c.label.long().cpu(), c.row_weight.double().cpu()
    g = torch.softmax(x @ w.T, 1)
    g[torch.arange(rows), label] -= 1.0
    g *= weight[:, None]
    own = torch.zeros_like(g)
    own[torch.arange(rows), label] = g[torch.arange(rows), label]
    others = g - own
    exact, half = g.T @ x, torch.finfo(c.t).eps / 2
    logit = (width / 4 + 32) * U32 * float((x.abs() @ w.abs().T).max())
    # (at once, the others are rounded twice; what was lost is at most half of the label's gradient, and its rounding half of that)
    tol = half * (1 + 2.0 ** -8) * exact.abs() + 2.02 * half * (others.abs().T @ x.abs()) + (half * half + 2 * logit + (rows / 4 + 64) * U32) * (g.abs().T @ x.abs()) \
        + TINY[type] + 2.0 ** (-39 if type == "float16" else -126) * 4 * float(weight.max()) * x.abs().sum(0)[None]
    for out in c.run(rk, ctx):
        bad = (out["d_weight"].double().cpu() - exact).abs() > tol
        assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[0].tolist())
