"""rk_route_forward / rk_route_backward against the definition in 64 bits.

Choices, counts and tokens are equal.  A probability is off by what its exponent is (the logit, its row's lse: each rounded to 32
bits a few times) and by the sum over at most 16 elements a lane and 64 lanes: TERMS times 2^-24 of p (1 + |l| + |lse|).
"""
import pytest

from oracle import training

pytestmark = pytest.mark.gpu
U32, TERMS = 2.0 ** -24, 64.0


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2408_08586_amd as rk
    ctx = rk.rk_create(0)
    yield torch, rk, ctx
    rk.rk_sync(ctx)
    rk.rk_destroy(ctx)


class Route:
    def __init__(self, gpu, logits, mask=None, top_k=2, renorm=True, group_tokens=0, pad=0):
        torch, self.rk, self.ctx = gpu
        self.torch = torch
        n, e = logits.shape
        self.logits = torch.full((n, e + pad), float("nan"), dtype=logits.dtype, device="cuda")[:, :e]
        self.logits.copy_(logits)
        self.mask = None if mask is None else mask.to(torch.uint8).cuda()
        self.n, self.e, self.k, self.renorm, self.group = n, e, top_k, renorm, group_tokens
        groups = (n + group_tokens - 1) // group_tokens if group_tokens else 1
        self.router = self.rk.make_router(e, top_k, renorm, group_tokens)
        f = lambda *s: torch.full(s, float("nan"), device="cuda")
        i = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")
        self.out = dict(expert=i(n, top_k), weight=f(n, top_k), lse=f(n), counts=i(groups, e), prob_sum=f(groups, e), tokens=i(groups), loss=f(2))

    def forward(self):
        self.rk.rk_route_forward(self.ctx, self.router, self.logits, self.mask, *self.out.values())
        return self.out

    def backward(self, d_loss, d_weight):
        torch, o = self.torch, self.out
        d = torch.full_like(self.logits, float("nan"))
        self.rk.rk_route_backward(self.ctx, self.router, self.logits, o["expert"], o["lse"], o["counts"], o["tokens"], d_loss.float().cuda(),
                                  None if d_weight is None else d_weight.float().cuda(), d)
        return d

    def check(self, seed=0, weights=True):
        torch = self.torch
        g = torch.Generator().manual_seed(seed)
        l = self.logits.double().cpu()
        mask = None if self.mask is None else self.mask.cpu()
        d_loss = torch.tensor([0.37, 0.11]).double()
        d_weight = torch.randn(self.n, self.k, generator=g).double() if weights else None
        d_weight = d_weight.float().double() if weights else None
        d_loss = d_loss.float().double()
        ref = training.route(l, mask, self.k, self.renorm, self.group, d_loss, d_weight)
        got = {k: v.cpu() for k, v in self.forward().items()}
        for name in ("expert", "counts", "tokens"):
            assert torch.equal(got[name].long(), ref[name].long()), name
        there = ref["there"]
        big = torch.where(there[:, None], l.abs().masked_fill(~torch.isfinite(l), 0.0), 0.0)
        row = 1 + big.max(1).values + ref["lse"].abs() if self.n else ref["lse"]
        near = lambda a, b, tol, what: self.near(a, b, tol, what)
        near(got["lse"], ref["lse"], TERMS * U32 * row, "lse")
        near(got["weight"], ref["weight"], TERMS * U32 * ref["weight"] * row[:, None], "weight")
        slack = U32 * (TERMS * row.max() + self.n) if self.n else U32
        near(got["prob_sum"], ref["prob_sum"], slack * ref["prob_sum"] + 1e-30, "prob_sum")
        near(got["loss"], ref["loss"], 2 * slack * ref["loss"] + 1e-30, "loss")
        d = self.backward(d_loss, d_weight).cpu()
        step = torch.finfo(d.dtype).eps / 2 if d.dtype != torch.float32 else 0.0
        tiny = 2.0 ** -25 if d.dtype == torch.float16 else 1e-37
        near(d, ref["d_logits"], step * (1 + 2.0 ** -8) * ref["d_logits"].abs() + 2 * TERMS * U32 * ref["big"] * row[:, None] + tiny, "d_logits")
        return ref

    def near(self, got, want, tol, what):
        bad = (got.double() - want).abs() > tol
        assert not bool(bad.any()) and not bool(self.torch.isnan(got).any()), \
            f"{what}: {int(bad.sum())} of {bad.numel()} beyond the tolerance at {bad.nonzero()[:1].tolist()}"


def logits_of(torch, n, e, dtype="float32", seed=0, spread=2.0):
    g = torch.Generator().manual_seed(seed * 131 + n * 7 + e)
    return (spread * torch.randn(n, e, generator=g)).to(getattr(torch, dtype))


@pytest.mark.parametrize("n", [1, 2, 5, 63, 130])
@pytest.mark.parametrize("e,k", [(1, 1), (2, 1), (3, 3), (8, 2), (16, 4), (31, 5), (60, 4), (64, 6), (65, 8), (128, 1), (160, 6), (256, 8), (257, 9), (300, 32), (512, 16), (1024, 8)])
def test_sizes(gpu, n, e, k):
    Route(gpu, logits_of(gpu[0], n, e), top_k=k, renorm=bool(n & 1)).check()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("group", [0, 1, 7, 40, 100, 1000])
def test_types_groups_and_masks(gpu, dtype, renorm, group):
    torch = gpu[0]
    mask = torch.rand(100, generator=torch.Generator().manual_seed(group)) > 0.3
    mask[40:80] = False                                  # whole groups without a token
    Route(gpu, logits_of(torch, 100, 72, dtype), mask, 4, renorm, group, pad=3).check()
    Route(gpu, logits_of(torch, 100, 72, dtype, seed=1), None, 4, renorm, group).check(weights=False)


@pytest.mark.parametrize("n,group", [(3000, 0), (9000, 1024), (20000, 20000)])
def test_many_tokens(gpu, n, group):
    Route(gpu, logits_of(gpu[0], n, 24, "bfloat16"), None, 3, True, group).check()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("e", [20, 64, 200, 1000])
def test_equal_logits_go_to_the_lowest_index(gpu, dtype, e):
    torch = gpu[0]
    l = torch.randint(-2, 3, (40, e), generator=torch.Generator().manual_seed(e)).to(getattr(torch, dtype))
    l[0] = 0.0
    l[1, ::2], l[1, 1::2] = 0.0, -0.0                    # zeros of both signs are equal
    l[2] = -l[2].abs()
    Route(gpu, l, None, min(8, e), True).check()


def test_logits_of_minus_infinity(gpu):
    """Fewer experts than are asked for, one, none; a masked token of infinities and NaN."""
    torch = gpu[0]
    l = logits_of(torch, 12, 48)
    l[1, 3:] = -float("inf")
    l[2, :] = -float("inf")
    l[2, 40] = 1.5
    l[3, :] = -float("inf")
    l[4, :24] = -float("inf")
    l[5, :], l[6, :] = float("nan"), float("inf")
    l[7, :] = torch.finfo(torch.float32).min
    l[8, 5:] = torch.finfo(torch.float32).min
    mask = torch.ones(12)
    mask[5] = mask[6] = 0
    for renorm in (False, True):
        r = Route(gpu, l, mask, 6, renorm)
        # (the lowest finite logits make lse as large: z is not looked at through these rows)
        l2 = l.clone()
        l2[7:9] = 0.0
        Route(gpu, l2, mask, 6, renorm).check()
        out = {k: v.cpu() for k, v in r.forward().items()}
        assert out["expert"][1].tolist()[3:] == [-1, -1, -1] and out["weight"][1, 3:].tolist() == [0, 0, 0]
        assert out["expert"][2].tolist() == [40, -1, -1, -1, -1, -1] and float(out["weight"][2, 0]) == 1.0
        for t in (3, 5, 6):
            assert out["expert"][t].tolist() == [-1] * 6 and float(out["lse"][t]) == 0.0
        assert out["expert"][7].tolist() == list(range(6))
        assert sorted(out["expert"][8].tolist()) == list(range(6)) and float(out["weight"][8, 5]) == 0.0
        assert int(out["tokens"][0]) == 9


def test_rows_that_are_not_finite_stay_alone(gpu):
    torch = gpu[0]
    l = logits_of(torch, 10, 64)
    clean = {k: v.clone() for k, v in Route(gpu, l, None, 4).forward().items()}
    l[4, 9], l[7, 30] = float("nan"), float("inf")
    got = Route(gpu, l, None, 4).forward()
    rest = [t for t in range(10) if t not in (4, 7)]
    for k in ("expert", "weight", "lse"):
        assert torch.equal(got[k][rest], clean[k][rest])
    assert bool(torch.isnan(got["weight"][4]).all()) and 9 not in got["expert"][4].tolist() and bool(torch.isnan(got["loss"]).all())


def test_no_tokens(gpu):
    for group in (0, 8):
        r = Route(gpu, logits_of(gpu[0], 0, 16), None, 2, True, group)
        out = r.forward()
        assert out["loss"].tolist() == [0.0, 0.0]
        if not group:
            assert out["counts"].tolist() == [[0] * 16] and out["tokens"].tolist() == [0]
        r.backward(gpu[0].zeros(2), None)
    r = Route(gpu, logits_of(gpu[0], 9, 16), gpu[0].zeros(9), 2)      # every token padding
    r.check()


def test_in_place(gpu):
    torch, rk, ctx = gpu
    r = Route(gpu, logits_of(torch, 70, 160, "bfloat16"), None, 6)
    o = r.forward()
    d_loss, dw = torch.tensor([0.1, 0.2]), torch.randn(70, 6)
    d = r.backward(d_loss, dw)
    rk.rk_route_backward(ctx, r.router, r.logits, o["expert"], o["lse"], o["counts"], o["tokens"], d_loss.cuda(), dw.cuda(), r.logits)
    assert torch.equal(d, r.logits)


def test_gradient_against_differences(gpu):
    torch = gpu[0]
    r = Route(gpu, logits_of(torch, 14, 20), None, 3, True, 5)
    ref = r.check()
    d_loss, dw = torch.tensor([0.37, 0.11]).double(), torch.randn(14, 3, generator=torch.Generator().manual_seed(0)).float().double()
    grad = r.backward(d_loss, dw).double().cpu()
    l, way = r.logits.double().cpu(), torch.randn(14, 20, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
    ends = []
    for h in (1e-5, -1e-5):
        out = training.route(l + h * way, None, 3, True, 5)
        assert torch.equal(out["expert"], ref["expert"])
        ends.append(float((d_loss * out["loss"]).sum() + (dw * out["weight"]).sum()))
    slope, formula = (ends[0] - ends[1]) / 2e-5, float((grad * way).sum())
    assert abs(slope - formula) <= 2e-5 * float((grad * way).abs().sum()) + 1e-7


def test_equal_calls_return_equal_bits_and_a_graph_replays_them(gpu):
    torch, rk, _ = gpu
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rk.rk_create(0)
        r = Route((torch, rk, ctx), logits_of(torch, 4000, 96, "bfloat16"), torch.rand(4000) > 0.2, 6, True, 1000)
        d_loss, dw, d = torch.tensor([0.1, 0.2], device="cuda"), torch.randn(4000, 6, device="cuda"), torch.empty_like(r.logits)
        o = r.out

        def step():
            r.forward()
            rk.rk_route_backward(ctx, r.router, r.logits, o["expert"], o["lse"], o["counts"], o["tokens"], d_loss, dw, d)

        everything = lambda: [t.clone() for t in (*o.values(), d)]
        step()
        first = everything()
        step()
        for a, b in zip(first, everything()):
            assert torch.equal(a, b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for turn in range(3):
            r.logits.mul_(1.125)
            graph.replay()
            replayed = everything()
            step()
            for a, b in zip(replayed, everything()):
                assert torch.equal(a, b), turn
        rk.rk_sync(ctx)
        rk.rk_destroy(ctx)
