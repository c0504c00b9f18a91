"""Sizes at which the recurrence and the vocabulary head go another way: tiles of 192 and 256 rows in 32 bits, several pieces of a
vocabulary in every type, tiles that hold whole sequences."""
import pytest

from test_gpu_head import TINY, U32, Case as Head, gpu  # noqa: F401  (fixture)
from test_gpu_recur import Case as Recur

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, vocab, width, ignored", [(300, 64000, 40, 0.2), (1000, 32000, 36, 0.1), (257, 65536, 33, 0.0)])
def test_large_tiles_in_32_bits(gpu, rows, vocab, width, ignored):
    """250 tiles of words, of 300 rows two turns of the card with 192 or 128 rows a tile: 192.  125 of 1,000 rows: 256 rows a tile.  The last tile of rows
    is cut short; loss and gradients apart and at once."""
    torch, rk, ctx = gpu
    Head(torch, rows, vocab, width, "float32", z=1e-3, ignored=ignored, seed=3).check(rk, ctx)


@pytest.mark.parametrize("type, weights", [("float16", False), ("float16", True), ("float32", False), ("float32", True)])
@pytest.mark.parametrize("width", [40, 33])
def test_several_pieces_in_every_type(gpu, type, weights, width):
    """More gradients than a piece holds, labels in every piece, the last word's and the first's among them: every element against 64 bits on the GPU.
    (At once, the last piece's elements in 16 bits are rounded twice, and for d_weight those of small weight.)"""
    torch, rk, ctx = gpu
    rows, vocab, t = 4200, 140001, getattr(torch, type)
    g = torch.Generator("cuda").manual_seed(width)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda").to(t)
    x, words = n(rows, width), n(vocab, width) * 0.5
    label = torch.randint(0, vocab, (rows,), generator=g, device="cuda").int()
    label[:3] = torch.tensor([0, vocab - 1, -1])
    f = lambda *s: torch.full(s, float("nan"), device="cuda")
    loss, lse, total, dx, dw = f(rows), f(rows), f(1), n(rows, width), n(vocab, width)
    row_weight = torch.exp2(torch.randint(-20, 1, (rows,), generator=g, device="cuda").float()) if weights else torch.ones(rows, device="cuda")
    given = (ctx, rk.make_head(), x, words, label, row_weight if weights else None)
    rk.rk_head_loss_backward(*given, None, loss, lse, total, dx, dw)
    dx2, dw2 = torch.empty_like(dx), torch.empty_like(dw)
    rk.rk_head_backward(*given, lse, None, dx2, dw2)
    double = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")
    w64 = words.double()
    exact = {"lse": double(rows), "loss": double(rows), "dx": double(rows, width), "dw": double(vocab, width)}
    size = {"dx": double(rows, width), "dw": double(vocab, width)}
    big = 0.0
    for a in range(0, rows, 700):
        part = slice(a, a + 700)
        x64, own, keep = x[part].double(), label[part].long(), label[part] >= 0
        l, at = x64 @ w64.t(), torch.arange(len(own), device="cuda")
        big = max(big, float((x64.abs() @ w64.abs().t()).max()))
        exact["lse"][part] = torch.where(keep, torch.logsumexp(l, 1), 0.0)
        exact["loss"][part] = torch.where(keep, torch.logsumexp(l, 1) - l[at, own.clamp(min=0)], 0.0)
        p = torch.softmax(l, 1)
        d = p.clone()
        d[at[keep], own[keep]] -= 1
        d[~keep], p[~keep] = 0, 0
        d, p = d * row_weight[part, None], p * row_weight[part, None]
        most = d.abs() + p
        exact["dx"][part], size["dx"][part] = d @ w64, most @ w64.abs()
        exact["dw"] += d.t() @ x64
        size["dw"] += most.t() @ x64.abs()
    # a logit: the number of its products over four and 32 units of their magnitudes; a probability: its logit's and its row's lse's error
    logit = (width / 4 + 32) * U32 * big
    p = 2 * logit + 64 * U32
    for got, want in ((lse, exact["lse"]), (loss, exact["loss"])):
        assert bool(((got.double() - want).abs() <= 2 * logit + 64 * U32 * (want.abs() + 1)).all())
    half = torch.finfo(t).eps / 2 if type != "float32" else 0.0
    # half of the smallest step of float16: of a 2^38th of the largest weight, of rows below a 64th of it of their own
    least = torch.where(row_weight >= 2.0 ** -6, 1.0, row_weight.double())[:, None]
    for times, which, name in ((2, dx, "dx"), (1, dx2, "dx"), (2, dw, "dw"), (2 if weights else 1, dw2, "dw")):
        other = (w64 if name == "dx" else x.double()).abs().sum(0)[None]
        steps = (vocab if name == "dx" else rows) / 4 + 64
        tol = (times * half + p + steps * U32) * size[name] + half * (1 + 2.0 ** -8) * exact[name].abs() + TINY[type] + 2.0 ** (-39 if type == "float16" else -126) * 4 * other * (least if name == "dx" else 1.0)
        bad = ~((which.double() - exact[name]).abs() <= tol)
        assert not bool(bad.any()), (name, times, int(bad.sum()), bad.nonzero()[0].tolist())


@pytest.mark.parametrize("type", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("seq_rows, rows, width, coupled", [(1, 300, 130, True), (1, 1030, 33, False), (64, 300, 129, True), (32, 700, 200, False), (128, 640, 64, True),
                                                            (4, 257, 1, True)])
def test_tiles_of_whole_sequences(gpu, type, seq_rows, rows, width, coupled):
    """Equal sequences that a tile of rows holds whole, in several tiles: no tile has anything to tell another.  (128 rows are a tile of 16 bits; of 32 bits
    two, and these tell.)"""
    torch, rk, ctx = gpu
    at = list(range(0, rows, seq_rows)) + [rows]
    for bias, states, pad in ((True, True, 0), (False, False, 5)):
        Recur(torch, at, width, uniform=seq_rows, type=type, coupled=coupled, bias=bias, states=states, pad=pad, seed=rows + width).check(rk, ctx)


def test_a_step_of_many_sequences_in_place(gpu):
    """Serving: one token of each of 300 sequences, three calls, the states carried in place; against the sequences in one call.  A row is a mean of x and the row
    before, so nothing is larger than the largest of x and the states, and row t of either is within 24 + 3 |v| units of t + 2 times that."""
    torch, rk, ctx = gpu
    n, steps, width = 300, 3, 70
    c = Recur(torch, [i * steps for i in range(n + 1)], width, type="float32", seed=21)
    h, state = c.forward(rk, ctx)
    now, recur = c.state_in.clone(), rk.Recur(bias=c.bias, seq_rows=1)
    unit = 2 * (24 + 3 * float((c.z + c.bias).abs().max())) * U32 * max(float(c.x.abs().max()), float(c.state_in.abs().max()))
    for t in range(steps):
        out = torch.empty(n, width, device="cuda")
        rk.rk_recur_forward(ctx, recur, c.x[t::steps], c.z[t::steps], now, out, now)
        assert float((out - h[t::steps]).abs().max()) <= unit * (t + 2)
    assert float((now - state).abs().max()) <= unit * (steps + 1)
