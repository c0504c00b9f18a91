"""The edges of what the header promises of recurrence and vocabulary head: the most sequences, rows whose weights are far apart."""
import pytest

from test_gpu_head import gpu  # noqa: F401  (fixture)

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
