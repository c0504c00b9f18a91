"""Rows of NaN, what a run that has diverged gives: they are no rows that were left out, and nothing hides them."""
import math

import pytest

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def gpu():
    import torch
    import paper_2408_08586_amd as rk
    ctx = rk.rk_create(0)
    yield torch, rk, ctx
    rk.rk_sync(ctx)
    rk.rk_destroy(ctx)


def test_oracle():
    import torch
    from oracle import training
    l = torch.zeros(4, 5, dtype=torch.float64)
    l[1], l[2], l[3] = NAN, -INF, -INF
    l[3, 2] = NAN
    r = training.route(l, None, 2, False, 0)
    assert r["there"].tolist() == [True, True, False, True] and float(r["tokens"][0]) == 3
    assert r["lse"].isnan().tolist() == [False, True, False, True] and bool(r["loss"].isnan().all())
    d = training.distill(l, l[:, :2], torch.tensor([[0, 1]] * 4), torch.zeros(4, dtype=torch.int64), None, 1.0, 0.5, 0.5)
    assert d["loss"].isnan().tolist() == [False, True, False, True] and float(d["lse"][2, 0]) == -INF


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("n", [12, 1500])
def test_routed_tokens_of_nan(gpu, dtype, renorm, n):
    from test_gpu_route import Route, logits_of
    torch = gpu[0]
    l = logits_of(torch, n, 48, dtype)
    mask = torch.ones(n)
    mask[9] = 0
    l[3], l[7], l[5], l[9] = NAN, -INF, -INF, NAN
    l[7, 11] = NAN                                       # beside nothing but -inf
    r = Route(gpu, l, mask, 4, renorm)
    out = {k: v.clone().cpu() for k, v in r.forward().items()}
    for t in (3, 7):
        assert out["expert"][t].tolist() == [-1] * 4 and math.isnan(float(out["lse"][t]))
    for t in (5, 9):
        assert out["expert"][t].tolist() == [-1] * 4 and out["weight"][t].tolist() == [0.0] * 4 and float(out["lse"][t]) == 0.0
    assert bool(torch.isnan(out["loss"]).all()) and int(out["tokens"][0]) == n - 2
    d = r.backward(torch.tensor([0.3, 0.2]), torch.ones(n, 4)).float().cpu()
    assert bool(torch.isnan(d[[3, 7]]).all()) and bool((d[[5, 9]] == 0).all())
    rest = [t for t in range(n) if t not in (3, 5, 7, 9)]
    clean = Route(gpu, torch.nan_to_num(l, nan=0.0, neginf=0.0), mask, 4, renorm).forward()
    for k in ("expert", "weight", "lse"):
        assert torch.equal(out[k][rest], clean[k][rest].cpu()), k


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("tau", [1.0, 2.0])
@pytest.mark.parametrize("rows,vocab", [(6, 700), (6, 20000), (300, 9000)])
def test_students_of_nan(gpu, dtype, tau, rows, vocab):
    from test_gpu_distill import Student
    torch = gpu[0]
    s = Student(gpu, rows, vocab, 5, dtype, kd=0.5, ce=0.5, weights=False, tau=tau)
    s.s[1], s.s[3], s.s[4] = NAN, -INF, -INF
    s.s[4, vocab // 2] = NAN
    out, d1, both, d2 = s.run()
    for o in (out, both):
        assert bool(torch.isnan(o["loss"][[1, 4]]).all()) and bool(torch.isnan(o["lse"][[1, 4]]).all()) and bool(torch.isnan(o["total"]).all())
        assert float(o["loss"][3]) == 0.0 and float(o["lse"][3, 0]) == -INF
    for d in (d1, d2):
        assert bool(torch.isnan(d[[1, 4]].float()).all()) and bool((d[3] == 0).all())
        assert bool(torch.isfinite(d[[0, 2, 5]].float()).all())
