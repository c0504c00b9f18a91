"""The edges of what the header promises of recurrence and vocabulary head: the most sequences, rows whose weights are far apart."""
import pytest

from oracle import training
from test_gpu_head import TINY, U32, Case as Head, gpu  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_seqs", [2 ** 30 - 1, 2 ** 30, 2 ** 31 - 3, 2 ** 31 - 2])
def test_as_many_sequences_as_there_may_be(gpu, n_seqs):
    """All of them without rows but two, the last and one in the middle: the rows are these two's, bit for bit what two sequences give."""
    torch, rk, ctx = gpu
    rows, width, cut = 300, 40, 170
    g = torch.Generator().manual_seed(1)
    x, z = (torch.randn(rows, width, generator=g).cuda() for _ in range(2))
    at = torch.zeros(n_seqs + 1, dtype=torch.int32, device="cuda")
    at[n_seqs // 2 + 1:], at[n_seqs:] = cut, rows
    few = torch.tensor([0, cut, rows], dtype=torch.int32, device="cuda")
    got = []
    for offsets in (at, few):
        recur = rk.Recur(offsets=offsets)
        h, dx, dz = (torch.full((rows, width), float("nan"), device="cuda") for _ in range(3))
        rk.rk_recur_forward(ctx, recur, x, z, None, h, None)
        rk.rk_recur_backward(ctx, recur, x, z, h, None, x, None, dx, dz, None, None)
        got.append((h, dx, dz))
    rk.rk_sync(ctx)
    assert all(torch.equal(a, b) and bool(torch.isfinite(b).all()) for a, b in zip(*got))


@pytest.mark.parametrize("z, d_total", [(0.0, 2.0 ** 16), (2.0, 2.0 ** 12)])
def test_float16_weights_of_very_different_rows(gpu, z, d_total):
    """float16 keeps a row's gradient of the logits down to 2^-32 of the row's own unit (for dx), and 2^-38 of the largest (for d_weight), whatever the
    other rows' weights are: a unit is a power of two, at or above |weight| max(1, |1 + 2 z lse|).  Both are rounded once or twice on the way, and what is
    smaller than a step by half of one."""
    torch, rk, ctx = gpu
    rows, vocab, width = 64, 300, 64
    c = Head(torch, rows, vocab, width, "float16", z=z, d_total=d_total, seed=5)
    c.row_weight = torch.exp2(torch.linspace(-32, -2, rows)).cuda()
    c.row_weight[::3] *= -1
    d = lambda t: t.double().cpu()
    x, w, weight = d(c.x), d(c.weight), d(c.row_weight)
    exact, size = training.head(x, w, c.label.cpu(), weight, 1.0, z, torch.tensor([d_total], dtype=torch.float64))
    half, p = torch.finfo(torch.float16).eps / 2, 2 * (width / 4 + 32) * U32 * float(size["big"].max()) + 64 * U32
    big = weight.abs() * (1 + 2 * z * exact["lse"]).abs().clamp(min=1.0)
    unit = torch.exp2(torch.ceil(torch.log2(big)))
    least = {"dx": 2.0 ** -33 * unit[:, None] * d_total * w.abs().sum(0)[None], "d_weight": 2.0 ** -39 * float(unit.max()) * d_total * x.abs().sum(0)[None]}
    for which, out in zip(("apart", "at once"), c.run(rk, ctx)):
        for k, steps in (("dx", vocab / 4 + 64), ("d_weight", rows / 4 + 64)):
            tol = (2 * half + p + steps * U32) * size[k] + half * (1 + 2.0 ** -8) * exact[k].abs() + TINY["float16"] + 1.01 * least[k]
            assert bool(torch.isfinite(out[k]).all())
            bad = ~((d(out[k]) - exact[k]).abs() <= tol)
            assert not bool(bad.any()), (which, k, int(bad.sum()), bad.nonzero()[0].tolist())


class Far:
    """Matrices side by side in rows that lie `stride` elements apart."""

    def __init__(self, torch, rows, stride, t):
        self.room, self.at = torch.empty(rows * stride, dtype=t, device="cuda").view(rows, stride), 0

    def __call__(self, v):
        self.at += 128
        return self.room[:v.shape[0], self.at - 128:self.at - 128 + v.shape[1]].copy_(v)


@pytest.mark.parametrize("type", ["bfloat16", "float32"])
def test_rows_beyond_2_to_32_elements(gpu, type):
    """Rows so far apart that the last begin beyond 2^32 elements: bit for bit what rows side by side give."""
    torch, rk, ctx = gpu
    t, rows, width = getattr(torch, type), 560, 72
    g = torch.Generator().manual_seed(3)
    n = lambda *s: torch.randn(*s, generator=g).to(t).cuda()
    near = lambda v: v.clone()
    x, z, dh = n(rows, width), n(rows, width), n(rows, width)
    recur = rk.Recur(bias=n(width), offsets=torch.tensor([0, 300, 300, rows], dtype=torch.int32, device="cuda"))
    got = []
    for at in (near, Far(torch, rows, 1 << 23, t)):
        h, dx, dz, db = at(x * 0), at(x * 0), at(x * 0), torch.empty(width, device="cuda")
        rk.rk_recur_forward(ctx, recur, at(x), at(z), None, h, None)
        rk.rk_recur_backward(ctx, recur, at(x), at(z), h, None, at(dh), None, dx, dz, None, db)
        got.append((h.clone(), dx.clone(), dz.clone(), db))
        rk.rk_sync(ctx)
    del at, h, dx, dz
    assert all(torch.equal(a, b) for a, b in zip(*got))
    # words of the head: so far apart that they are padded first, and less far
    for vocab, stride in ((560, 1 << 23), (1 << 14, 1 << 19)):
        words, label, got = n(vocab, width), torch.randint(0, vocab, (90,), generator=g).int().cuda(), []
        for at in (near, Far(torch, vocab, stride, t)):
            f = lambda *s: torch.full(s, float("nan"), device="cuda")
            dx, dw, loss, lse, total = at(x[:90] * 0), at(words * 0), f(90), f(90), f(1)
            rk.rk_head_loss_backward(ctx, rk.make_head(), at(x[:90]), at(words), label, None, None, loss, lse, total, dx, dw)
            got.append((dx.clone(), dw.clone(), loss, lse, total))
            rk.rk_sync(ctx)
        del at, dx, dw
        assert all(torch.equal(a, b) and bool(torch.isfinite(a).all()) for a, b in zip(*got))
    torch.cuda.empty_cache()
