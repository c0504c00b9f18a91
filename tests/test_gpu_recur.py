"""rk_recur_forward / rk_recur_backward against the recurrence in 64 bits, row after row.

Tolerance of an element: half a step of its type, and 2^-24 of its size (oracle.training: what an error of one unit of every row's magnitude
adds up to on its way) times STEP + 3 |v|: a gate's exponential is off by |v| log2(e) of half a step of its exponent and two of its own, the
sum, the quotient and the products of a row by one or two each, twelve at most, and twice that where a run of rows
is first taken by itself and then joined with what came before.
"""
import numpy as np
import pytest

from oracle import training

pytestmark = pytest.mark.gpu
U32, STEP = 2.0 ** -24, 24.0
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


def close(torch, got, exact, size, what, units, rows=None):
    g, e, s = got.double().cpu(), exact, size
    name = str(got.dtype)[6:]
    tol = (torch.finfo(got.dtype).eps / 2 if name != "float32" else 0.0) * e.abs() * (1 + 2.0 ** -8) + units * U32 * s + TINY[name]
    bad = ~((g - e).abs() <= tol) & ~((torch.isnan(g) & torch.isnan(e)) | (g == e))
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} beyond the tolerance, the first at {bad.nonzero()[0].tolist()}: "
                                 f"{float(g[bad][0])!r} instead of {float(e[bad][0])!r} +- {float(tol[bad][0]):.2e}")


class Case:
    def __init__(self, torch, at, width, rows=None, type="bfloat16", params=None, coupled=True, bias=True, states=True, pad=0, off=0, seed=0,
                 uniform=None, shift=1.0, spread=1.5):
        g = torch.Generator().manual_seed(seed * 131 + width)
        self.torch, self.at, self.width, self.rows = torch, at, width, rows or at[-1]
        self.t, self.pad, self.off, self.coupled, self.uniform = getattr(torch, type), pad, off, coupled, uniform
        n = lambda *s: torch.randn(*s, generator=g)
        self.x, self.dh = self.matrix(n(self.rows, width)), self.matrix(0.1 * n(self.rows, width))
        self.z = self.matrix(spread * n(self.rows, width) + (0.0 if bias else shift))
        self.bias = (shift + n(width)).to(getattr(torch, params or type)).cuda() if bias else None
        self.state_in = self.state(n(len(at) - 1, width)) if states else None
        self.d_state_out = self.state(0.1 * n(len(at) - 1, width)) if states else None

    def matrix(self, values=None):
        """Rows `pad` elements apart, the first `off` elements behind an aligned address, NaN between them."""
        torch, stride = self.torch, self.width + self.pad
        room = torch.full((self.rows * stride + self.off + 8,), float("nan"), dtype=self.t, device="cuda")
        m = room[self.off:self.off + self.rows * stride].view(self.rows, stride)[:, :self.width]
        return m if values is None else m.copy_(values)

    def state(self, values=None):
        torch = self.torch
        room = torch.full((max(1, len(self.at) - 1), self.width + self.pad % 3), float("nan"), device="cuda")[:len(self.at) - 1, :self.width]
        return room if values is None else room.copy_(values)

    def recur(self, rk):
        how = {"seq_rows": self.uniform} if self.uniform is not None else \
            {"offsets": self.torch.tensor(self.at, dtype=self.torch.int32, device="cuda")}
        return rk.Recur(coupled=self.coupled, bias=self.bias, **how)

    def forward(self, rk, ctx):
        h, state = self.matrix(), self.state() if self.state_in is not None else None
        rk.rk_recur_forward(ctx, self.recur(rk), self.x, self.z, self.state_in, h, state)
        return h, state

    def backward(self, rk, ctx, h):
        dx, dz = self.matrix(), self.matrix()
        dsi = self.state() if self.state_in is not None else None
        db = self.torch.full((self.width,), float("nan"), device="cuda") if self.bias is not None else None
        rk.rk_recur_backward(ctx, self.recur(rk), self.x if self.coupled else None, self.z, h, self.state_in, self.dh, self.d_state_out, dx, dz, dsi, db)
        return dx, dz, dsi, db

    def check(self, rk, ctx):
        torch = self.torch
        h, state = self.forward(rk, ctx)
        dx, dz, dsi, db = self.backward(rk, ctx, h)
        d = lambda t: None if t is None else t.double().cpu()
        out, size = training.recurrence(d(self.x), d(self.z), d(self.bias), self.at, self.coupled, d(self.state_in), d(self.dh), d(self.d_state_out), d(h))
        v = d(self.z) + (d(self.bias) if self.bias is not None else 0.0)
        units = STEP + 3 * float(v.abs().nan_to_num(0.0).max()) if v.numel() else STEP
        close(torch, h, out["h"], size["h"], "h", units)
        close(torch, dx, out["dx"], size["dx"], "dx", units)
        close(torch, dz, out["dz"], size["dz"], "dz", units)
        if state is not None:
            close(torch, state, out["state_out"], size["state_out"], "state_out", units)
            close(torch, dsi, out["d_state_in"], size["d_state_in"], "d_state_in", units)
        if db is not None:                                  # (sums of eight rows, eight wavefronts, a sixteenth of the tiles of 64 rows, sixteen runs)
            close(torch, db, out["d_bias"], size["d_bias"], "d_bias", units + 32 + self.rows / 1024)


RAGGED = [0, 0, 1, 2, 2, 2, 19, 83, 84, 84, 211, 300, 301, 301]


@pytest.mark.parametrize("type", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("coupled", [True, False])
def test_ragged(gpu, type, coupled):
    torch, rk, ctx = gpu
    for width, pad, off, params in ((70, 0, 0, None), (1, 2, 1, "float32"), (257, 3, 1, None), (512, 8, 0, "float32")):
        Case(torch, RAGGED, width, type=type, coupled=coupled, pad=pad, off=off, params=params, seed=width).check(rk, ctx)


@pytest.mark.parametrize("at", [[0, 1], [0, 2], [0, 15, 16], [0, 16, 33], [0, 63, 64, 65], [0, 129], [0, 500, 1000], [0, 2049], list(range(201)),
                                [0, 0, 0], [0, 0, 700], [0, 700, 700]])
def test_lengths(gpu, at):
    torch, rk, ctx = gpu
    for bias, states in ((True, True), (False, False)):
        Case(torch, at, 40, bias=bias, states=states, seed=len(at)).check(rk, ctx)


@pytest.mark.parametrize("seq_rows, rows", [(0, 300), (300, 300), (1, 40), (7, 100), (128, 512), (100, 512), (1000, 300), (256, 257)])
def test_equal_lengths(gpu, seq_rows, rows):
    torch, rk, ctx = gpu
    at = [0, rows] if not seq_rows else list(range(0, rows, seq_rows)) + [rows]
    Case(torch, at, 130, uniform=seq_rows, type="float32", seed=rows).check(rk, ctx)


@pytest.mark.parametrize("type", ["bfloat16", "float32"])
def test_a_long_sequence(gpu, type):
    """Long enough for many tiles of rows, one behind the other; gates that remember for thousands of rows."""
    torch, rk, ctx = gpu
    Case(torch, [0, 12001], 33, type=type, shift=6.0, spread=1.0, states=True, seed=5).check(rk, ctx)
    Case(torch, [0, 5000, 5001, 9000], 300, type=type, shift=5.0, spread=0.5, bias=False, seed=6).check(rk, ctx)


def test_rows_that_no_sequence_has(gpu):
    """Before the first and behind the last sequence nothing is read or written."""
    torch, rk, ctx = gpu
    c = Case(torch, [5, 9, 200], 64, rows=400, type="float32", seed=8)
    for m in (c.x, c.z, c.dh):
        m[:5], m[200:] = float("nan"), float("nan")
    c.check(rk, ctx)                                        # (what is left as it was is NaN on both sides)


def test_a_nan_stays_in_its_sequence(gpu):
    torch, rk, ctx = gpu
    at = [0, 100, 300, 420]
    c = Case(torch, at, 64, type="float32", seed=9)
    c.x[150, 3], c.z[160, 5], c.x[170, 7], c.z[110, 9], c.z[111, 10] = float("nan"), float("nan"), float("inf"), float("inf"), -float("inf")
    c.state_in[1, 11] = float("nan")
    h, state = c.forward(rk, ctx)
    clean = Case(torch, at, 64, type="float32", seed=9)
    h0, state0 = clean.forward(rk, ctx)
    other = [r for r in range(420) if not 100 <= r < 300]
    assert torch.equal(h[other], h0[other]) and torch.equal(state[[0, 2]], state0[[0, 2]])
    assert bool(torch.isnan(h[150:300, 3]).all()) and bool(torch.isnan(h[160:300, 5]).all()) and bool(torch.isinf(h[170, 7]))
    assert bool(torch.isnan(h[100:300, 11]).all()) and bool(torch.isnan(state[1, [3, 5, 11]]).all())
    # a gate that is fully open keeps the state, one that is closed takes x
    assert torch.equal(h[110, 9], h[109, 9]) and torch.equal(h[111, 10], c.x[111, 10])
    c.dh[250, 20] = float("nan")
    dx, dz, dsi, db = c.backward(rk, ctx, h0)
    dx0, dz0, dsi0, db0 = clean.backward(rk, ctx, h0)
    assert torch.equal(dx[other], dx0[other]) and torch.equal(dsi[[0, 2]], dsi0[[0, 2]])
    assert bool(torch.isnan(dx[100:251, 20]).all()) and not bool(torch.isnan(dx[251:300, 20]).any()) and bool(torch.isnan(dsi[1, 20]))


def test_in_place(gpu):
    torch, rk, ctx = gpu
    for at in (RAGGED, [0, 3000], list(range(65))):
        c = Case(torch, at, 200, seed=11)
        h, state = c.forward(rk, ctx)
        dx, dz, dsi, db = c.backward(rk, ctx, h)
        for into in ("x", "z"):
            d = Case(torch, at, 200, seed=11)
            rk.rk_recur_forward(ctx, d.recur(rk), d.x, d.z, d.state_in, getattr(d, into), d.state_in)
            assert torch.equal(getattr(d, into), h) and torch.equal(d.state_in, state)
        d = Case(torch, at, 200, seed=11)
        dz2, dsi2, db2 = d.matrix(), d.state(), torch.empty_like(db)
        rk.rk_recur_backward(ctx, d.recur(rk), d.x, d.z, h, d.state_in, d.dh, d.d_state_out, d.dh, dz2, dsi2, db2)
        assert torch.equal(d.dh, dx) and torch.equal(dz2, dz) and torch.equal(dsi2, dsi) and torch.equal(db2, db)


def test_step_by_step_is_the_whole(gpu):
    """Serving: a token of every sequence a call, states carried along in place, against the sequences in one call (the state is float32 in both)."""
    torch, rk, ctx = gpu
    n, steps, width = 9, 20, 96
    c = Case(torch, [i * steps for i in range(n + 1)], width, type="float32", seed=12)
    h, state = c.forward(rk, ctx)
    now = c.state_in.clone()
    recur = rk.Recur(bias=c.bias, seq_rows=1)
    for t in range(steps):
        x, z, out = c.x[t::steps], c.z[t::steps], torch.empty(n, width, device="cuda")
        rk.rk_recur_forward(ctx, recur, x, z, now, out, now)
        assert torch.allclose(out, h[t::steps], rtol=1e-5, atol=1e-6)
    assert torch.allclose(now, state, rtol=1e-5, atol=1e-6)


def test_equal_calls_return_equal_bits(gpu):
    torch, rk, ctx = gpu
    c = Case(torch, [0, 3000, 3001, 7000], 600, seed=13)
    h, state = c.forward(rk, ctx)
    first = c.backward(rk, ctx, h)
    for _ in range(5):
        again = c.forward(rk, ctx)
        assert torch.equal(again[0], h) and torch.equal(again[1], state)
        assert all(torch.equal(a, b) for a, b in zip(c.backward(rk, ctx, h), first))


def test_in_a_graph(gpu):
    """Captured on its own stream and replayed with other inputs, eager calls of other shapes on the context between the replays."""
    torch, rk, _ = gpu
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rk.rk_create(0)
        c = Case(torch, [0, 1500, 1500, 2600], 300, seed=14)
        other = Case(torch, [0, 700], 100, seed=15)
        recur = c.recur(rk)
        h, state, dx, dz, dsi, db = c.matrix(), c.state(), c.matrix(), c.matrix(), c.state(), torch.empty(300, device="cuda")

        def both():
            rk.rk_recur_forward(ctx, recur, c.x, c.z, c.state_in, h, state)
            rk.rk_recur_backward(ctx, recur, c.x, c.z, h, c.state_in, c.dh, c.d_state_out, dx, dz, dsi, db)

        both()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            both()
        for i in range(4):
            c.x.copy_(c.x.float() * 0.9 + 0.05 * i)
            c.z.copy_(c.z.float() * 0.95)
            both()
            want = [t.clone() for t in (h, state, dx, dz, dsi, db)]
            for t in (h, state, dx, dz, dsi, db):
                t.zero_()
            other.forward(rk, ctx)
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((h, state, dx, dz, dsi, db), want)), i
        rk.rk_sync(ctx)
        rk.rk_destroy(ctx)


def test_gradients_are_differences(gpu):
    """In 32 bits, a few directions of x, z, bias and state against central differences of the loss; the kernel's own forward pass."""
    torch, rk, ctx = gpu
    c = Case(torch, [0, 5, 5, 40], 12, type="float32", seed=16)
    h, state = c.forward(rk, ctx)
    dx, dz, dsi, db = c.backward(rk, ctx, h)

    def loss():
        h, state = c.forward(rk, ctx)
        return float((h.double() * c.dh.double()).sum() + (state.double() * c.d_state_out.double()).sum())

    g = torch.Generator().manual_seed(1)
    for what, grad in ((c.x, dx), (c.z, dz), (c.bias, db), (c.state_in, dsi)):
        way, keep = torch.randn(what.shape, generator=g).cuda(), what.clone()
        eps = 2.0 ** -6
        what.copy_(keep + eps * way)
        up = loss()
        what.copy_(keep - eps * way)
        down = loss()
        what.copy_(keep)
        slope, want = (up - down) / (2 * eps), float((grad.double() * way.double()).sum())
        # the differences' third-order term, and the loss's rounding over the step
        scale = float((grad.double() * way.double()).abs().sum())
        assert abs(slope - want) <= 4 * eps ** 2 * scale + 1e-5 / eps * 0.1, (slope, want)


def test_no_sequences(gpu):
    """Offsets that hold no sequence, and rows without any: nothing is written but the bias's gradient of zero."""
    torch, rk, ctx = gpu
    for rows in (0, 5):
        f = lambda *s: torch.full(s, float("nan"), device="cuda")
        x, recur = torch.randn(rows, 33, device="cuda"), rk.Recur(bias=torch.zeros(33, device="cuda"), offsets=torch.zeros(1, dtype=torch.int32, device="cuda"))
        h, state, dx, dz, db = f(rows, 33), f(0, 33), f(rows, 33), f(rows, 33), f(33)
        rk.rk_recur_forward(ctx, recur, x, x, state, h, state)
        rk.rk_recur_backward(ctx, recur, x, x, h, None, x, None, dx, dz, None, db)
        assert bool(torch.isnan(h).all()) and bool(torch.isnan(dx).all()) and bool((db == 0).all())
    # rows without a sequence length end are one sequence, also of no rows: its state goes through
    state, out = torch.randn(1, 33, device="cuda"), f(1, 33)
    e = torch.empty(0, 33, device="cuda")
    rk.rk_recur_forward(ctx, rk.Recur(), e, e, state, e, out)
    assert torch.equal(out, state)
    # a length beyond any number of rows is one sequence
    x = torch.randn(200, 34, device="cuda")
    a, b = f(200, 34), f(200, 34)
    rk.rk_recur_forward(ctx, rk.Recur(seq_rows=2 ** 64 - 1), x, x, None, a, None)
    rk.rk_recur_forward(ctx, rk.Recur(), x, x, None, b, None)
    assert torch.equal(a, b)


def test_offsets_that_are_none_lead_nowhere(gpu):
    """Descending, negative and far offsets: the results are nobody's business, but the call ends and writes no other rows' memory."""
    torch, rk, ctx = gpu
    rows, width = 400, 66
    room = torch.zeros(rows + 2, width, device="cuda")
    x = torch.randn(rows, width, device="cuda")
    for at in ([300, 100, 200, 50, 400], [-7, 30, 1000000, 60], [2 ** 31 - 1, -2 ** 31, 0, 400], [5, 5, 4, 5, 399]):
        recur = rk.Recur(offsets=torch.tensor(at, dtype=torch.int32, device="cuda"))
        n = len(at) - 1
        states = torch.zeros(n + 2, width, device="cuda")
        h, d = room[1:rows + 1], torch.empty(rows, width, device="cuda")
        rk.rk_recur_forward(ctx, recur, x, x, torch.zeros(n, width, device="cuda"), h, states[1:n + 1])
        rk.rk_recur_backward(ctx, recur, x, x, h, None, x, torch.zeros(n, width, device="cuda"), torch.empty_like(d), d, torch.zeros(n, width, device="cuda"), None)
        rk.rk_sync(ctx)
        assert bool((room[0] == 0).all()) and bool((room[-1] == 0).all()) and bool((states[0] == 0).all()) and bool((states[-1] == 0).all())
