"""rk_dropout_forward / rk_dropout_backward against Philox in whole numbers and the sum in 64 bits.

Which elements stay is compared exactly.  What stays is off by half a step of its type, and in 32 bits by the roundings of the
scale, the product and the sum, a unit of 2^-24 each."""
import pytest

from oracle import training

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


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


def rng_of(torch, seed, offset):
    signed = lambda v: v - 2 ** 64 if v >= 2 ** 63 else v
    return torch.tensor([signed(seed), signed(offset)], dtype=torch.int64, device="cuda")


TYPES = ("bfloat16", "float16", "float32")


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("rows, width, pad, off, p", [(1, 1, 0, 0, 0.5), (3, 7, 0, 0, 0.25), (5, 8, 0, 0, 0.1), (17, 65, 2, 1, 0.3), (2, 1000, 0, 0, 0.9),
                                                       (40, 24, 8, 0, 0.5), (3, 333, 3, 3, 0.0), (4, 50, 0, 1, 1.0), (1, 4111, 0, 0, 1e-4)])
def test_against_whole_numbers(gpu, type, wide, rows, width, pad, off, p):
    torch, rk, ctx = gpu
    t, r = getattr(torch, type), torch.float32 if wide else getattr(torch, type)
    g = torch.Generator().manual_seed(rows * width)
    seed, offset = 0x9123456789ABCDEF ^ rows, 0xF000000500000003 + width
    d = rk.Dropout(p, rng_of(torch, seed, offset))
    least = int(float(torch.tensor(p, dtype=torch.float32)) * 65536 + 0.5)
    keep = training.dropout_numbers(range(rows), width, seed, offset) >= least
    scale = 65536.0 / (65536 - least) if least < 65536 else 0.0
    x = room(torch, rows, width, t, pad, off, torch.randn(rows, width, generator=g) + 3.0)
    residual = room(torch, rows, width, r, pad, off, torch.randn(rows, width, generator=g))
    for res in (residual, None):
        out = room(torch, rows, width, r, pad, off)
        rk.rk_dropout_forward(ctx, d, x, res, out)
        before = res.double().cpu() if res is not None else torch.zeros(rows, width, dtype=torch.float64)
        value = torch.where(keep, x.double().cpu() * scale, 0.0)
        exact, got = before + value, out.double().cpu()
        assert torch.equal(got[~keep], before[~keep])
        tol = (torch.finfo(r).eps / 2 if r != torch.float32 else 0.0) * exact.abs() * (1 + 2.0 ** -8) + 3 * U32 * (value.abs() + before.abs()) + 2.0 ** -25 * (r == torch.float16)
        assert bool(((got - exact).abs() <= tol).all())
    d_out = room(torch, rows, width, r, pad, off, torch.randn(rows, width, generator=g) + 3.0)
    dx = room(torch, rows, width, t, pad, off)
    rk.rk_dropout_backward(ctx, d, d_out, dx)
    exact, got = torch.where(keep, d_out.double().cpu() * scale, 0.0), dx.double().cpu()
    assert bool((got[~keep] == 0).all())
    assert bool(((got - exact).abs() <= (torch.finfo(t).eps / 2 + 3 * U32) * exact.abs() * (1 + 2.0 ** -8) + 2.0 ** -25 * (t == torch.float16)).all())


def test_the_mask_is_the_elements_own(gpu):
    """Strides, types and directions do not change which elements stay; the offset and the seed do; the rows before do not."""
    torch, rk, ctx = gpu
    rows, width = 300, 517
    ones = lambda t, pad: room(torch, rows, width, t, pad, pad % 2, torch.ones(rows, width))
    masks = []
    d = rk.Dropout(0.4, rng_of(torch, 77, 5))
    for t, pad in ((torch.bfloat16, 0), (torch.float16, 3), (torch.float32, 8)):
        out = ones(t, pad)
        rk.rk_dropout_forward(ctx, d, ones(t, pad), None, out)
        masks.append(out != 0)
        rk.rk_dropout_backward(ctx, d, ones(t, pad), out)
        masks.append(out != 0)
    assert all(torch.equal(m, masks[0]) for m in masks)
    out = torch.empty(7, width, device="cuda")
    rk.rk_dropout_forward(ctx, d, torch.ones(7, width, device="cuda"), None, out)
    assert torch.equal(out != 0, masks[0][:7])
    for seed, offset in ((77, 6), (78, 5), (77 + 2 ** 32, 5), (77, 5 + 2 ** 32)):
        rk.rk_dropout_forward(ctx, rk.Dropout(0.4, rng_of(torch, seed, offset)), ones(torch.float32, 0), None, out := ones(torch.float32, 0))
        differ = float(((out != 0) != masks[0]).float().mean())
        assert 0.46 < differ < 0.50                         # 2 x 0.4 x 0.6 of 155,100: 0.48 +- 0.0013
    share = float(masks[0].float().mean())
    assert abs(share - 0.6) < 0.007                         # five deviations: sqrt(0.24 / 155100) x 5


def test_what_is_dropped_leaves_nothing(gpu):
    torch, rk, ctx = gpu
    d = rk.Dropout(0.5, rng_of(torch, 1, 1))
    x, res, out = torch.full((64, 200), float("nan"), device="cuda"), torch.full((64, 200), 2.0, device="cuda"), torch.empty(64, 200, device="cuda")
    x[::2] = float("inf")
    rk.rk_dropout_forward(ctx, d, x, res, out)
    assert bool(((out == 2.0) | ~torch.isfinite(out)).all()) and 0.4 < float((out == 2.0).float().mean()) < 0.6
    every = rk.Dropout(1.0, rng_of(torch, 1, 1))
    rk.rk_dropout_forward(ctx, every, x, res, out)
    assert bool((out == 2.0).all())


def test_in_place_and_many_rows(gpu):
    torch, rk, ctx = gpu
    for rows, width, t in ((3, 100003, torch.bfloat16), (70001, 40, torch.float16), (2049, 777, torch.float32)):
        x, res = torch.randn(rows, width, device="cuda").to(t), torch.randn(rows, width, device="cuda").to(t)
        d = rk.Dropout(0.1, rng_of(torch, 3, 9))
        out = torch.empty_like(x)
        rk.rk_dropout_forward(ctx, d, x, res, out)
        y, r = x.clone(), res.clone()
        rk.rk_dropout_forward(ctx, d, y, r, y)
        rk.rk_dropout_forward(ctx, d, x, r, r)
        assert torch.equal(y, out) and torch.equal(r, out)
        rk.rk_dropout_backward(ctx, d, x, out)
        y = x.clone()
        rk.rk_dropout_backward(ctx, d, y, y)
        assert torch.equal(y, out)
        some = sorted({0, 1, rows // 2, rows - 1})
        numbers = training.dropout_numbers(some, min(width, 4001), 3, 9).cuda()
        kept = numbers >= 6554
        assert torch.equal(out[some][:, :kept.shape[1]] != 0, kept & (x[some][:, :kept.shape[1]] != 0))


def test_replays_take_the_state_of_their_time(gpu):
    torch, rk, _ = gpu
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rk.rk_create(0)
        rng = rng_of(torch, 11, 0)
        d = rk.Dropout(0.5, rng)
        x, out = torch.ones(50, 333, device="cuda"), torch.empty(50, 333, device="cuda")
        rk.rk_dropout_forward(ctx, d, x, None, out)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            rk.rk_dropout_forward(ctx, d, x, None, out)
            rng[1:].add_(1)
        seen = []
        for i in range(4):
            rng[1] = i
            rk.rk_dropout_forward(ctx, d, x, None, out)
            want = out.clone()
            out.zero_()
            graph.replay()
            stream.synchronize()
            assert torch.equal(out, want) and int(rng[1]) == i + 1
            seen.append(want)
        assert not torch.equal(seen[0], seen[1])
        rk.rk_sync(ctx)
        rk.rk_destroy(ctx)


def test_no_rows(gpu):
    torch, rk, ctx = gpu
    e = torch.empty(0, 5, device="cuda")
    rk.rk_dropout_forward(ctx, rk.Dropout(0.5, rng_of(torch, 1, 1)), e, None, torch.empty(0, 5, device="cuda"))
