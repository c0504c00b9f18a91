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
