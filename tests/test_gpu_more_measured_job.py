"""Recurrence, dropout and head together, as the example that measures a job uses them."""
import os
import sys

import numpy as np
import pytest

from oracle import training

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import measure_job
    return measure_job


def test_a_run_with_all_of_them(example):
    m = example.measure(256, 64, 2, layers=2, experts=4, vocab=500, kept=16, steps=4, recurrence=True, dropout=0.1, head=True)
    assert np.isfinite(m["history"]).all() and m["forward"] > 0 and m["backward"] > 0
    # without logits the forward keeps less, though the recurrence keeps its own
    other = example.measure(256, 64, 2, layers=2, experts=4, vocab=500, kept=16, steps=4, recurrence=True, dropout=0.1)
    assert m["bytes_kept"] < other["bytes_kept"] and m["params_layers"] == other["params_layers"] and m["params_rest"] == other["params_rest"]


def test_the_command(example):
    m, records = example.main(["--params", "1e8", "--layers", "12", "--seq", "128", "--vocab", "1000", "--steps", "2", "--recurrence", "--dropout", "0.2", "--head"])
    assert int(records["g"].sum()) <= 8 and np.isfinite(m["history"]).all()


def test_gradients_of_a_chain(example):
    """Products, recurrence, dropout onto the stream, head: in 32 bits, every gradient against torch's of the same chain in 64 bits under the
    mask that the counters give.  Three products of 48 and one of 200 in a row, each off by 2^-24 times its length over four and eight units more,
    gates by 24 units (a row's memory sums these over some ten rows): of what the gradients' magnitudes are, 2^-24 x 2000 is more than all of that."""
    import torch
    import paper_2408_08586_amd as rk
    torch.backends.cuda.matmul.allow_tf32 = False
    ctx = rk.rk_create(0)
    rows, width, vocab, seq, p = 90, 48, 200, 30, 0.3
    g = torch.Generator().manual_seed(7)
    n = lambda *s: torch.randn(*s, generator=g)
    host = {"dense": n(width, width) / width ** 0.5, "forget": n(width, width) / width ** 0.5, "bias": 1.0 + 0.3 * n(width), "words": n(vocab, width) / width ** 0.5}
    x, label = n(rows, width), torch.randint(0, vocab, (rows,), generator=g)
    dev = {k: v.cuda().requires_grad_() for k, v in host.items()}
    xd = x.cuda()
    drop = rk.Dropout(p, torch.tensor([31, 4], device="cuda"))
    y = example.Recurrence.apply(ctx, xd @ dev["dense"], xd @ dev["forget"], dev["bias"], seq)
    u = xd + example.Drop.apply(ctx, drop, y)
    f = lambda *s: torch.empty(*s, device="cuda")
    weight, total, loss, lse = torch.full((rows,), 1 / rows, device="cuda"), f(1), f(rows), f(rows)
    du, dev["words"].grad = f(rows, width), f(vocab, width)
    rk.rk_head_loss_backward(ctx, rk.make_head(z_weight=1e-3), u.detach(), dev["words"].detach(), label.int().cuda(), weight, None, loss, lse, total, du, dev["words"].grad)
    u.backward(du)

    keep = (training.dropout_numbers(range(rows), width, 31, 4) >= round(p * 65536)).double() * 65536 / (65536 - round(p * 65536))
    double = {k: v.double().requires_grad_() for k, v in host.items()}
    xs = x.double()
    v, forget = xs @ double["dense"], torch.sigmoid(xs @ double["forget"] + double["bias"])
    hidden = []
    for t in range(rows):
        h = torch.zeros(width, dtype=torch.float64) if t % seq == 0 else hidden[-1]
        hidden.append(forget[t] * h + (1 - forget[t]) * v[t])
    logits = (xs + torch.stack(hidden) * keep) @ double["words"].t()
    z = torch.logsumexp(logits, 1)
    want = (z - logits[torch.arange(rows), label] + 1e-3 * z ** 2).mean()
    want.backward()
    assert abs(float(total) - float(want)) <= 2000 * 2.0 ** -24 * float(want)
    for k in host:
        a, b = dev[k].grad.double().cpu(), double[k].grad
        assert float((a - b).abs().max()) <= 2000 * 2.0 ** -24 * float(b.abs().max()), k
    rk.rk_sync(ctx)
    rk.rk_destroy(ctx)


def test_a_step_in_a_graph_on_another_stream(example):
    """Two contexts on two streams, their steps captured and replayed side by side: each has its own working buffers."""
    import torch
    import paper_2408_08586_amd as rk
    rows, width, vocab = 300, 96, 700
    sides = []
    for i in range(2):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            g = torch.Generator().manual_seed(i)
            n = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()
            s = {"ctx": rk.rk_create(0), "stream": stream, "x": n(rows, width), "z": n(rows, width), "words": (n(vocab, width) * 0.1), "res": n(rows, width),
                 "label": torch.randint(0, vocab, (rows,), generator=g).int().cuda(), "recur": rk.Recur(seq_rows=150), "drop": rk.Dropout(0.2, torch.tensor([i, 0], device="cuda")),
                 "head": rk.make_head()}
            e = lambda *k, t=torch.bfloat16: torch.empty(*k, dtype=t, device="cuda")
            s["out"] = {"h": e(rows, width), "u": e(rows, width), "loss": e(rows, t=torch.float32), "lse": e(rows, t=torch.float32), "total": e(1, t=torch.float32),
                        "du": e(rows, width), "dw": e(vocab, width), "dh": e(rows, width), "dx": e(rows, width), "dz": e(rows, width)}

            def step(s=s):
                o = s["out"]
                rk.rk_recur_forward(s["ctx"], s["recur"], s["x"], s["z"], None, o["h"], None)
                rk.rk_dropout_forward(s["ctx"], s["drop"], o["h"], s["res"], o["u"])
                rk.rk_head_loss_backward(s["ctx"], s["head"], o["u"], s["words"], s["label"], None, None, o["loss"], o["lse"], o["total"], o["du"], o["dw"])
                rk.rk_dropout_backward(s["ctx"], s["drop"], o["du"], o["dh"])
                rk.rk_recur_backward(s["ctx"], s["recur"], s["x"], s["z"], o["h"], None, o["dh"], None, o["dx"], o["dz"], None, None)

            s["step"] = step
            step()
            stream.synchronize()
            s["graph"] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(s["graph"], stream=stream):
                step()
            stream.synchronize()
            sides.append(s)
    for turn in range(4):
        wants = []
        for s in sides:
            with torch.cuda.stream(s["stream"]):
                s["x"].mul_(0.9)
                s["step"]()
                wants.append({k: v.clone() for k, v in s["out"].items()})
                for v in s["out"].values():
                    v.zero_()
        torch.cuda.synchronize()
        for s in sides:
            with torch.cuda.stream(s["stream"]):
                s["graph"].replay()
        torch.cuda.synchronize()
        for s, want in zip(sides, wants):
            assert all(torch.equal(s["out"][k], want[k]) for k in want), turn
    for s in sides:
        rk.rk_sync(s["ctx"])
        rk.rk_destroy(s["ctx"])
