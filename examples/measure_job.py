"""A job's descriptor, measured: a few layers of a mixture-of-experts student are trained for some steps on this GPU, and what the
steps take and keep becomes the t_fwd_sample, k_bwd and mem_act that a scheduling round is then run with.

    python examples/measure_job.py [--params 1.3e9] [--layers 24] [--experts 8] [--steps 8]

The products are torch's; what lies between them are the library's operators: the join of each block with the residual stream
(rk_norm_forward / rk_norm_backward), the router (rk_route_forward / rk_route_backward) and the student's loss
(rk_distill_loss_backward).  Data and weights are random.  A layer is a dense block and a block of experts, without attention, and the
job that is scheduled is this very student: its width follows from --params, its parameters are counted, and what its layers take is scaled to
all of them, while the first norm, the output's product and the loss count once.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2408_08586_amd as rk  # noqa: E402
import workloads  # noqa: E402

DEV = "cuda:0"
BALANCE, ROUTER_Z = 0.01, 0.001                         # weights of the router's two losses


def f32(*shape):
    return torch.empty(*shape, dtype=torch.float32, device=DEV)


def i32(*shape):
    return torch.empty(*shape, dtype=torch.int32, device=DEV)


class Join(torch.autograd.Function):
    """(stream, block's output) -> (stream, next block's input); post_weight None: the stream's first norm, without a block."""

    @staticmethod
    def forward(fn, ctx, x, y, post_weight, pre_weight, gate):
        block = rk.NormBlock(post="none" if y is None else "rms", pre="rms", post_weight=post_weight, pre_weight=pre_weight, gate=gate)
        x_out, u, stats = torch.empty_like(x), torch.empty_like(x), f32(x.shape[0], 4)
        rk.rk_norm_forward(ctx, block, x, y, x_out, u, stats)
        fn.ctx, fn.block = ctx, block
        fn.save_for_backward(x_out, y, stats)
        return x_out, u

    @staticmethod
    def backward(fn, dx_out, du):
        x_out, y, stats = fn.saved_tensors
        grads = rk.NormGrads(fn.block)
        dx, dy = torch.empty_like(x_out), None if y is None else torch.empty_like(y)
        rk.rk_norm_backward(fn.ctx, fn.block, x_out, y, stats, dx_out.contiguous(), du.contiguous(), dx, dy, grads)
        g = grads.tensors
        return None, dx, dy, g.get("post_weight"), g["pre_weight"], g.get("gate")


class Route(torch.autograd.Function):
    """logits -> (weights, experts, losses [balance, z])."""

    @staticmethod
    def forward(fn, ctx, router, logits):
        n, k, e = logits.shape[0], router.top_k, router.n_experts
        groups = (n + router.group_tokens - 1) // router.group_tokens if router.group_tokens else 1
        expert, weight, lse, counts = i32(n, k), f32(n, k), f32(n), i32(groups, e)
        tokens, loss = i32(groups), f32(2)
        rk.rk_route_forward(ctx, router, logits, None, expert, weight, lse, counts, f32(groups, e), tokens, loss)
        fn.ctx, fn.router = ctx, router
        fn.save_for_backward(logits, expert, lse, counts, tokens)
        fn.mark_non_differentiable(expert)
        return weight, expert, loss

    @staticmethod
    def backward(fn, d_weight, _, d_loss):
        logits, expert, lse, counts, tokens = fn.saved_tensors
        d_logits = torch.empty_like(logits)
        rk.rk_route_backward(fn.ctx, fn.router, logits, expert, lse, counts, tokens, d_loss.contiguous(), d_weight.contiguous(), d_logits)
        return None, None, d_logits


class Student:
    """`layers` layers of a dense block and a block of experts, norms in float32 and products in bfloat16."""

    def __init__(self, hidden, layers, experts, top_k, vocab, seq, seed=0):
        g = torch.Generator(DEV).manual_seed(seed)
        self.router = rk.make_router(experts, top_k, renormalise=True, group_tokens=seq)
        self.layers, self.params = layers, {}

        def product(name, *shape):
            w = torch.randn(*shape, generator=g, device=DEV) / shape[-2] ** 0.5
            self.params[name] = w.to(torch.bfloat16).requires_grad_()

        def vector(name, value, *shape):
            self.params[name] = torch.full(shape, value, device=DEV, requires_grad=True)

        vector("first", 1.0, hidden)
        for i in range(layers):
            product(f"dense{i}", hidden, hidden)
            product(f"router{i}", hidden, experts)
            product(f"up{i}", experts, hidden, hidden)
            product(f"down{i}", experts, hidden, hidden)
            for b in ("a", "b"):
                vector(f"post{b}{i}", 1.0, hidden)
                vector(f"pre{b}{i}", 1.0, hidden)
                vector(f"gate{b}{i}", 0.5, 1, hidden)
        product("head", hidden, vocab)
        count = {n: p.numel() for n, p in self.params.items()}
        self.params_rest = count["first"] + count["head"]
        self.params_layers = sum(count.values()) - self.params_rest

    def experts(self, i, u, weight, expert):
        """Every expert's product on the tokens that chose it, a copy a choice, put back in the tokens' order.  (How many chose it comes to
        the host, a wait in every layer that is part of what this student takes.)"""
        k = expert.shape[1]
        order = torch.argsort(expert.reshape(-1), stable=True)
        sizes = torch.bincount(expert.reshape(-1), minlength=self.router.n_experts).tolist()
        parts = []
        for e, rows in enumerate(torch.split(u[order // k], sizes)):
            up = torch.nn.functional.silu(rows @ self.params[f"up{i}"][e])
            parts.append(up @ self.params[f"down{i}"][e])
        back = torch.empty_like(order)
        back[order] = torch.arange(len(order), device=DEV)
        return (torch.cat(parts)[back].view(-1, k, u.shape[1]) * weight[:, :, None]).sum(1).to(torch.bfloat16)

    def forward(self, ctx, x, mark=lambda where, u: None):
        """mark is called with the input of the first layer and the output of the last."""
        p, losses = self.params, []
        x, u = Join.apply(ctx, x, None, None, p["first"], None)
        mark("layers", u)
        for i in range(self.layers):
            y = u @ p[f"dense{i}"]
            x, u = Join.apply(ctx, x, y, p[f"posta{i}"], p[f"prea{i}"], p[f"gatea{i}"])
            weight, expert, loss = Route.apply(ctx, self.router, u @ p[f"router{i}"])
            losses.append(loss)
            x, u = Join.apply(ctx, x, self.experts(i, u, weight, expert), p[f"postb{i}"], p[f"preb{i}"], p[f"gateb{i}"])
        mark("head", u)
        return u @ p["head"], losses


def measure(hidden, seq, micro_batch, layers=2, experts=8, top_k=2, vocab=32000, kept=64, steps=8, rate=1e-3, seed=0):
    """Trains for `steps` steps; seconds forward and backward of one, bytes that the forward keeps, each also of the layers alone, the
    student's parameters, and the losses by step."""
    ctx = rk.rk_create(0)
    student = Student(hidden, layers, experts, top_k, vocab, seq, seed)
    g = torch.Generator(DEV).manual_seed(seed + 1)
    tokens = seq * micro_batch
    x = torch.randn(tokens, hidden, generator=g, device=DEV).to(torch.bfloat16)
    label = torch.randint(0, vocab, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    # a teacher that is mostly sure of the label
    index = torch.stack([(label + j * 17) % vocab for j in range(kept)], 1).to(torch.int32)
    teacher = torch.linspace(4.0, -2.0, kept, device=DEV).expand(tokens, kept).contiguous()
    distill = rk.make_distill(temperature=2.0, kd_weight=0.5, ce_weight=0.5)
    row_weight = torch.full((tokens,), 1.0 / tokens, device=DEV)
    loss, lse, total = f32(tokens), f32(tokens, 2), f32(1)
    d_losses = torch.tensor([BALANCE, ROUTER_Z], device=DEV)
    times, history, kept_at = [], [], {}
    for step in range(steps):
        torch.cuda.synchronize()
        ev = {n: torch.cuda.Event(enable_timing=True) for n in ("start", "layers", "head", "forward", "back_head", "back_layers", "backward")}

        def mark(where, u):
            ev[where].record()
            kept_at[where] = torch.cuda.memory_allocated()
            # (the gradient of what a layer gets is there when all behind it has gone back)
            u.register_hook(lambda _: ev["back_head" if where == "head" else "back_layers"].record())

        before = torch.cuda.memory_allocated()
        ev["start"].record()
        logits, losses = student.forward(ctx, x, mark)
        ev["forward"].record()
        kept_at["forward"] = torch.cuda.memory_allocated()
        d_logits = torch.empty_like(logits)
        rk.rk_distill_loss_backward(ctx, distill, logits.detach(), teacher, index, label, row_weight, None, loss, lse, total, d_logits)
        torch.autograd.backward([logits] + losses, [d_logits] + [d_losses] * len(losses))
        ev["backward"].record()
        with torch.no_grad():
            for p in student.params.values():
                p -= rate * torch.sign(p.grad)
                p.grad = None
        torch.cuda.synchronize()
        took = lambda a, b: ev[a].elapsed_time(ev[b]) * 1e-3
        times.append((took("start", "forward"), took("layers", "head"), took("forward", "backward"), took("back_head", "back_layers")))
        history.append((float(total), sum(float(l.detach()[0]) for l in losses) / len(losses)))
        del logits, losses, d_logits                    # (the next step's forward is not to find them where it counts what it keeps)
    rk.rk_sync(ctx)
    rk.rk_destroy(ctx)
    forward, forward_layers, backward, backward_layers = (float(t) for t in np.median(np.array(times[1:] or times), axis=0))
    return dict(forward=forward, forward_layers=forward_layers, backward=backward, backward_layers=backward_layers,
                bytes_kept=int(kept_at["forward"] - before), bytes_layers=int(kept_at["head"] - kept_at["layers"]),
                params_layers=student.params_layers, params_rest=student.params_rest, history=history)


def descriptor(workload, job, m, layers, seq, micro_batch):
    """The workload's job with what was measured in place of its drawn coefficients: what the layers take, keep and are is scaled to all
    of the job's layers, what is outside them counts once (what it keeps, at the measured micro-batch, is part of the constant)."""
    coef, ints = workload.coef.copy(), workload.ints.copy()
    col = {n: i for i, n in enumerate(workloads.COEF_FIELDS)}
    times, hidden = float(ints[job, 0]) / layers, float(coef[job, col["hidden"]])
    forward = m["forward"] + m["forward_layers"] * (times - 1)
    backward = m["backward"] + m["backward_layers"] * (times - 1)
    coef[job, col["P_bytes"]] = 2 * (m["params_layers"] * times + m["params_rest"])
    coef[job, col["t_fwd_sample"]] = forward / micro_batch
    coef[job, col["k_bwd"]] = max(1.0, backward / forward)
    coef[job, col["mem_act"]] = m["bytes_layers"] / (seq * micro_batch * hidden * layers)
    coef[job, col["mem_const"]] += m["bytes_kept"] - m["bytes_layers"]
    return coef, ints


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    a.add_argument("--params", type=float, default=1.3e9)
    a.add_argument("--layers", type=int, default=24)
    a.add_argument("--measured-layers", type=int, default=2)
    a.add_argument("--experts", type=int, default=8)
    a.add_argument("--seq", type=int, default=2048)
    a.add_argument("--vocab", type=int, default=32000)
    a.add_argument("--steps", type=int, default=8)
    a = a.parse_args(argv)
    # params ~ layers (1 + 2 experts) h^2 + vocab h
    per = a.layers * (1 + 2 * a.experts)
    hidden = 128 * max(1, round(((a.vocab ** 2 + 4 * per * a.params) ** 0.5 - a.vocab) / (2 * per) / 128))
    m = measure(hidden, a.seq, 1, a.measured_layers, a.experts, vocab=a.vocab, steps=a.steps)
    for step, (total, balance) in enumerate(m["history"]):
        print(f"step {step}: loss {total:.4f}, balance {balance:.4f}")
    print(f"{a.measured_layers} layers of {hidden}: forward {m['forward'] * 1e3:.2f} ms, backward {m['backward'] * 1e3:.2f} ms, "
          f"{m['bytes_kept'] / 2 ** 20:.0f} MiB kept; of the layers alone {m['forward_layers'] * 1e3:.2f} and {m['backward_layers'] * 1e3:.2f} ms, "
          f"{m['bytes_layers'] / 2 ** 20:.0f} MiB")
    wl = workloads.tiny()
    col = {n: i for i, n in enumerate(workloads.COEF_FIELDS)}
    wl.coef[0, [col["hidden"], col["seq"]]] = hidden, a.seq
    wl.ints[0] = (a.layers, 32, 1)
    coef, ints = descriptor(wl, 0, m, a.measured_layers, a.seq, 1)
    coef, ints = coef[:1], ints[:1]                     # the job alone on one node
    print(f"{coef[0, col['P_bytes']] / 2e9:.2f} billion parameters, t_fwd_sample {coef[0, col['t_fwd_sample']]:.4f} s, k_bwd {coef[0, col['k_bwd']]:.2f}, mem_act {coef[0, col['mem_act']]:.1f}")
    ctx = rk.rk_create(0)
    jobs = rk.Jobs(coef, ints)
    assign, total = rk.new_assign(1), torch.zeros(1, device=DEV)
    rk.rk_schedule_round(ctx, jobs, rk.make_bounds(wl.bounds), rk.make_grid(wl.grid), rk.make_env(wl.env), rk.make_cluster(wl.cluster), assign, total)
    rk.rk_sync(ctx)
    records = rk.assign_to_numpy(assign)
    rk.rk_destroy(ctx)
    print("on a node of 8 GPUs the round gives it", dict(zip(records.dtype.names, records[0].tolist())))
    return m, records


if __name__ == "__main__":
    main()
