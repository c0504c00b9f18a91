"""The example that measures a job: the operators together, trained for some steps, and the round that is run with what was measured."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import measure_job
    return measure_job


def test_a_few_steps_learn(example):
    m = example.measure(256, 64, 2, layers=2, experts=4, top_k=2, vocab=500, kept=16, steps=10, rate=2e-3)
    first, last = m["history"][0], m["history"][-1]
    assert np.isfinite(m["history"]).all()
    assert last[0] < 0.7 * first[0]                     # the student follows its teacher
    assert 0.9 < last[1] < 4.0                          # balance lies between 1 (even) and the number of experts
    assert m["forward"] > 0 and m["backward"] > 0 and m["bytes_kept"] > 0


def test_gradients_of_the_whole_step(example):
    """The step's gradient along a random direction of all its float32 vectors against differences of the loss.  The products and their
    inputs are bfloat16: a loss of size 1 over 64 rows moves by parts in 2^9 of what a row adds, so the step is large."""
    import torch
    import paper_2408_08586_amd as rk
    ctx = rk.rk_create(0)
    s = example.Student(128, 1, 4, 4, 96, 32, seed=3)   # every expert is chosen: nothing jumps
    g = torch.Generator("cuda").manual_seed(5)
    x = torch.randn(64, 128, generator=g, device="cuda").to(torch.bfloat16)
    label = torch.randint(0, 96, (64,), generator=g, device="cuda", dtype=torch.int32)
    distill, w = rk.make_distill(1.0, 0.0, 1.0), torch.full((64,), 1 / 64, device="cuda")
    loss, lse, total = example.f32(64), example.f32(64, 2), example.f32(1)

    def value():
        logits, losses = s.forward(ctx, x)
        d = torch.empty_like(logits)
        rk.rk_distill_loss_backward(ctx, distill, logits.detach(), None, None, label, w, None, loss, lse, total, d)
        return logits, d, float(total)

    logits, d, _ = value()
    logits.backward(d)
    names = [n for n, p in s.params.items() if p.dtype == torch.float32]
    ways = {n: torch.randn(s.params[n].shape, generator=g, device="cuda") for n in names}
    slope = sum(float((s.params[n].grad * ways[n]).sum()) for n in names)
    h, ends = 0.02, []
    for sign in (1, -1):
        with torch.no_grad():
            for n in names:
                s.params[n] += sign * h * ways[n]
            ends.append(value()[2])
            for n in names:
                s.params[n] -= sign * h * ways[n]
    size = sum(float((s.params[n].grad * ways[n]).abs().sum()) for n in names)
    assert abs((ends[0] - ends[1]) / (2 * h) - slope) <= 0.05 * size + 2 ** -9 / h / 8
    rk.rk_sync(ctx)
    rk.rk_destroy(ctx)


def test_the_measured_descriptor_is_scheduled(example):
    m, records = example.main(["--params", "1e8", "--layers", "12", "--seq", "128", "--vocab", "1000", "--steps", "3"])
    assert int(records["g"].sum()) <= 8 and float(records["thr"][0]) >= 0.0
    assert int(records["g"][0]) > 0                     # one GPU holds it
