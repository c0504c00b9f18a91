"""The operators of a training step in 64 bits, plainly, with the magnitudes that their errors are measured against.

Test infrastructure only.  Every function takes float64 tensors (the values that the operator is given, exactly) and returns the
results by name together with, for each, the sum of the magnitudes that enter it: an operator in 32 bits is off by a small
multiple of 2^-24 of that, whatever cancels.
"""
from __future__ import annotations

import torch

INF = float("inf")


def _vec(v, like, none):
    return torch.full_like(like[:1], none) if v is None else v.reshape(1, -1) if v.dim() == 1 else v


def _gates(gate, gate_rows, like):
    if gate is None:
        return torch.ones_like(like)
    if not gate_rows:
        return gate.expand_as(like)
    return gate[torch.arange(like.shape[0], device=like.device) // gate_rows]


def _stats(v, how, eps):
    rows = v.shape[0]
    if how == "none":
        return v.new_zeros(rows, 1), v.new_ones(rows, 1)
    mean = v.mean(1, keepdim=True) if how == "layer" else v.new_zeros(rows, 1)
    return mean, 1.0 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + eps)


def norm_forward(x, y, post, pre, vec, gate_rows, res_scale, post_eps, pre_eps):
    """vec: post_weight, post_bias, pre_weight, pre_bias, gate by name (or absent)."""
    g = _gates(vec.get("gate"), gate_rows, x)
    w1, b1 = _vec(vec.get("post_weight"), x, 1.0), _vec(vec.get("post_bias"), x, 0.0)
    w2, b2 = _vec(vec.get("pre_weight"), x, 1.0), _vec(vec.get("pre_bias"), x, 0.0)
    if y is None:
        my, ry = x.new_zeros(x.shape[0], 1), x.new_ones(x.shape[0], 1)
        xo, big = res_scale * x, (res_scale * x).abs()
    else:
        my, ry = _stats(y, post, post_eps)
        xo = res_scale * x + g * ((y - my) * ry * w1 + b1)
        big = (res_scale * x).abs() + g.abs() * ((y.abs() + my.abs()) * ry * w1.abs() + b1.abs())
    mx, rx = _stats(xo, pre, pre_eps)
    u = (xo - mx) * rx * w2 + b2
    # a mean is off by its row's magnitudes, 1/sqrt(..) relatively
    row = big.mean(1, keepdim=True)
    size = {"x_out": big, "u": (big + row + mx.abs()) * rx * w2.abs() + b2.abs(),
            "stats": torch.cat([t for v, m, r in ((y if y is not None else x, my, ry), (xo, mx, rx))
                                for t in (v.abs().mean(1, keepdim=True), r * (1 + r * big.mean(1, keepdim=True) * (v is xo)))], 1)}
    return {"x_out": xo, "u": u, "stats": torch.cat((my, ry, mx, rx), 1)}, size


def norm_backward(xo, y, stats, dxo, du, post, pre, vec, gate_rows, res_scale):
    rows = xo.shape[0]
    g = _gates(vec.get("gate"), gate_rows, xo)
    w1, b1 = _vec(vec.get("post_weight"), xo, 1.0), _vec(vec.get("post_bias"), xo, 0.0)
    w2 = _vec(vec.get("pre_weight"), xo, 1.0)
    my, ry, mx, rx = (stats[:, i:i + 1] for i in range(4))
    dxo = torch.zeros_like(xo) if dxo is None else dxo
    out, size = {}, {}

    def through(f, big_f, v, mean, r, how):
        hat, big_hat = (v - mean) * r, (v.abs() + mean.abs()) * r
        if how == "none":
            return f, big_f, hat, big_hat
        d = f - hat * (f * hat).mean(1, keepdim=True)
        big = big_f + big_hat * (big_f * big_hat).mean(1, keepdim=True)
        if how == "layer":
            d, big = d - f.mean(1, keepdim=True), big + big_f.mean(1, keepdim=True)
        return r * d, r * big, hat, big_hat

    d, big = dxo, dxo.abs()
    if pre != "none":
        e = du * w2
        t, b, hat, big_hat = through(e, e.abs(), xo, mx, rx, pre)
        d, big = d + t, big + b
        out["pre_weight"], size["pre_weight"] = (du * hat).sum(0), (du.abs() * big_hat).sum(0)
        out["pre_bias"], size["pre_bias"] = du.sum(0), du.abs().sum(0)
    out["dx"], size["dx"] = res_scale * d, abs(res_scale) * big
    if y is not None:
        dn, big_dn = d * g, big * g.abs()
        f, big_f = dn * w1, big_dn * w1.abs()
        out["dy"], size["dy"], hat, big_hat = through(f, big_f, y, my, ry, post)
        out["post_weight"], size["post_weight"] = (dn * hat).sum(0), (big_dn * big_hat).sum(0)
        out["post_bias"], size["post_bias"] = dn.sum(0), big_dn.sum(0)
        dg, big_g = d * (hat * w1 + b1), big * (big_hat * w1.abs() + b1.abs())
        per = gate_rows or max(rows, 1)
        stack = lambda v: torch.stack([p.sum(0) for p in torch.split(v, per)]) if rows else v.new_zeros(0 if gate_rows else 1, v.shape[1])
        out["gate"], size["gate"] = stack(dg), stack(big_g)
    return out, size


def route(logits, mask, top_k, renormalise, group_tokens, d_loss=None, d_weight=None):
    """Everything of both directions, token by token in the definition's words."""
    n_tok, n_exp = logits.shape
    per = group_tokens or max(n_tok, 1)
    groups = (n_tok + per - 1) // per if group_tokens else 1
    there = ~(logits == -INF).all(1) if n_tok else torch.zeros(0, dtype=torch.bool)
    if mask is not None:
        there = there & (mask != 0)
    p = torch.zeros_like(logits)
    lse = logits.new_zeros(n_tok)
    expert = torch.full((n_tok, top_k), -1, dtype=torch.int64)
    weight = logits.new_zeros(n_tok, top_k)
    counts, prob_sum = logits.new_zeros(groups, n_exp), logits.new_zeros(groups, n_exp)
    tokens = logits.new_zeros(groups)
    for t in range(n_tok):
        if not there[t]:
            continue
        l = logits[t]
        top = l.nan_to_num(nan=-INF, posinf=INF, neginf=-INF).max()
        lse[t] = top + torch.log(torch.exp(l - top).sum())
        p[t] = torch.exp(l - lse[t])
        order = sorted((e for e in range(n_exp) if float(l[e]) > -INF), key=lambda e: (-float(l[e]), e))[:top_k]
        expert[t, :len(order)] = torch.tensor(order)
        weight[t, :len(order)] = p[t, order]
        if renormalise:
            weight[t, :len(order)] = weight[t, :len(order)] / weight[t].sum()
        g = t // per
        counts[g, order] += 1
        prob_sum[g] += p[t]
        tokens[g] += 1
    used = tokens > 0
    n_used, n = int(used.sum()), float(tokens.sum())
    scale = torch.where(used, n_exp / (top_k * tokens.clamp(min=1) ** 2) / max(n_used, 1), 0.0)
    loss = torch.stack(((scale[:, None] * counts * prob_sum).sum(), (lse ** 2).sum() / max(n, 1.0)))
    out = dict(there=there, p=p, expert=expert, weight=weight, lse=lse, counts=counts, prob_sum=prob_sum, tokens=tokens, loss=loss)
    if d_loss is None:
        return out
    d, big = torch.zeros_like(logits), torch.zeros_like(logits)
    d_weight = torch.zeros_like(weight) if d_weight is None else d_weight
    for t in range(n_tok):
        if not there[t]:
            continue
        a = d_loss[0] * scale[t // per] * counts[t // per]
        x, on = torch.zeros_like(a), torch.zeros_like(a)
        for k in range(top_k):
            if expert[t, k] >= 0:
                x[expert[t, k]], on[expert[t, k]] = d_weight[t, k], 1.0
        z = d_loss[1] * 2 * lse[t] / max(n, 1.0)
        b = a if renormalise else a + x
        d[t] = p[t] * (b - (b * p[t]).sum() + z)
        big[t] = p[t] * (b.abs() + (b.abs() * p[t]).sum() + z.abs())
        if renormalise:
            w = on * p[t] / (on * p[t]).sum()
            d[t] += w * (x - (w * x).sum())
            big[t] += w * (x.abs() + (w * x.abs()).sum())
    out.update(d_logits=d, big=big)
    return out


def distill(student, t_logits, index, label, row_weight, tau, kd, ce, d_total=1.0):
    rows, vocab = student.shape
    loss, big_loss = student.new_zeros(rows), student.new_zeros(rows)
    lse, d, big = student.new_zeros(rows, 2), torch.zeros_like(student), torch.zeros_like(student)
    for r in range(rows):
        w = 1.0 if row_weight is None else float(row_weight[r])
        if w == 0.0:
            continue
        s = student[r]
        if bool((s == -INF).all()):
            lse[r] = torch.tensor([-INF if kd else 0.0, -INF if ce else 0.0])
            continue
        top = s.nan_to_num(nan=-INF, posinf=INF, neginf=-INF).max()
        if kd:
            lse[r, 0] = top / tau + torch.log(torch.exp((s - top) / tau).sum())
            kept = [k for k in range(index.shape[1]) if 0 <= int(index[r, k]) < vocab and float(t_logits[r, k]) != -INF]
            if kept:
                at, t = index[r, kept].long(), t_logits[r, kept] / tau
                log_q = t - t.max() - torch.log(torch.exp(t - t.max()).sum())
                q, log_p = torch.exp(log_q), s[at] / tau - lse[r, 0]
                some = q > 0
                loss[r] += kd * tau ** 2 * (q * (log_q - log_p))[some].sum()
                big_loss[r] += kd * tau ** 2 * (q * (log_q.abs() + (s[at] / tau).abs() + lse[r, 0].abs() + top.abs() / tau + 1))[some].sum()
                p = torch.exp(s / tau - lse[r, 0])
                f = kd * tau * w * d_total
                d[r] += f * (p - torch.zeros_like(s).index_add(0, at, q))
                big[r] += abs(f) * (p * (1 + (s / tau).abs() + lse[r, 0].abs()) + torch.zeros_like(s).index_add(0, at, q * (1 + log_q.abs() + t.abs())))
        if ce:
            lse[r, 1] = top + torch.log(torch.exp(s - top).sum())
            c = int(label[r])
            if 0 <= c < vocab:
                loss[r] += ce * (lse[r, 1] - s[c])
                big_loss[r] += ce * (lse[r, 1].abs() + s[c].abs() + top.abs() + 1)
                p = torch.exp(s - lse[r, 1])
                hot = torch.zeros_like(s)
                hot[c] = 1.0
                d[r] += ce * w * d_total * (p - hot)
                big[r] += abs(ce * w * d_total) * (p * (1 + s.abs() + lse[r, 1].abs()) + hot)
    wv = torch.ones(rows, dtype=torch.float64) if row_weight is None else row_weight
    total = torch.where(wv != 0, wv * loss, 0.0).sum().reshape(1)
    big = torch.nan_to_num(big, nan=0.0)
    return dict(loss=loss, lse=lse, total=total, d_student=d, big_loss=big_loss, big=big)
