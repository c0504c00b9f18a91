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


# ---------------------------------------------------------------------- gated recurrence
def recurrence(x, z, bias, at, coupled, state_in, dh=None, d_state_out=None, h_given=None):
    """Rows of sequences at[i] .. at[i + 1] - 1, one after the other.  Sizes: what an error of one unit of each row's own magnitude adds up
    to on its way through the rows behind it.  With dh, the gradients too, from h as given; rows that no sequence has are NaN."""
    n, width = len(at) - 1, z.shape[1]
    v = z if bias is None else z + bias
    f, nf = torch.sigmoid(v), torch.sigmoid(-v)
    share = nf if coupled else torch.ones_like(nf)
    start = torch.zeros(n, width, dtype=torch.float64) if state_in is None else state_in.clone()
    nan = lambda *s: torch.full(s, float("nan"), dtype=torch.float64)
    out, size = {"h": nan(*z.shape), "state_out": start.clone()}, {"h": nan(*z.shape), "state_out": start.abs()}
    for s in range(n):
        h, big, err = start[s], start[s].abs(), start[s].abs()
        for t in range(at[s], at[s + 1]):
            h = f[t] * h + share[t] * x[t]
            big = f[t] * big + share[t] * x[t].abs()
            err = f[t] * err + big
            out["h"][t], size["h"][t] = h, err
        out["state_out"][s], size["state_out"][s] = h, err
    if dh is None:
        return out, size
    before = nan(*z.shape)
    back = torch.zeros(n, width, dtype=torch.float64) if d_state_out is None else d_state_out
    names = ("dx", "dz")
    for k in names:
        out[k], size[k] = nan(*z.shape), nan(*z.shape)
    out["d_state_in"], size["d_state_in"] = back.clone(), back.abs()
    out["d_bias"], size["d_bias"] = torch.zeros(width, dtype=torch.float64), torch.zeros(width, dtype=torch.float64)
    for s in range(n):
        carry, big, err = back[s], back[s].abs(), back[s].abs()
        for t in reversed(range(at[s], at[s + 1])):
            before[t] = h_given[t - 1] if t > at[s] else start[s]
            e, big = dh[t] + carry, dh[t].abs() + big
            err = err + big
            of = before[t] - x[t] if coupled else before[t]
            most = before[t].abs() + (x[t].abs() if coupled else 0.0)
            out["dx"][t], size["dx"][t] = share[t] * e, share[t] * err
            out["dz"][t], size["dz"][t] = e * of * f[t] * nf[t], err * most * f[t] * nf[t]
            out["d_bias"] += out["dz"][t]
            size["d_bias"] += size["dz"][t]
            carry, big, err = f[t] * e, f[t] * big, f[t] * err
        out["d_state_in"][s], size["d_state_in"][s] = carry, err
    return out, size


# ---------------------------------------------------------------------- dropout
def philox(counter, key):
    """Philox4x32-10 (Salmon, Moraes, Dror and Shaw, 2011) of one counter, in whole numbers."""
    c, k, low = list(counter), list(key), 0xFFFFFFFF
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & low, (p >> 32) ^ c[3] ^ k[1], p & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def dropout_numbers(rows, width, seed, offset):
    """The 16-bit number of every element: rows is a list of row numbers."""
    low = 0xFFFFFFFF
    out = torch.empty(len(rows), (width + 7) // 8 * 8, dtype=torch.int32)
    for i, r in enumerate(rows):
        for g in range((width + 7) // 8):
            words = philox((g, r, offset & low, offset >> 32), (seed & low, seed >> 32))
            out[i, 8 * g:8 * g + 8] = torch.tensor([w >> s & 0xFFFF for w in words for s in (0, 16)], dtype=torch.int32)
    return out[:, :width]


# ---------------------------------------------------------------------- vocabulary head
def head(x, weight, label, row_weight, scale, z_weight, d_total, lse_given=None):
    """Loss, lse, total and gradients; sizes: of the logits (loss, lse), and the magnitudes that the gradients' sums take in: g |W| and g |x|."""
    rows, vocab = x.shape[0], weight.shape[0]
    w = torch.ones(rows, dtype=torch.float64) if row_weight is None else row_weight
    there = (w != 0) & (label >= 0) & (label < vocab)
    kept = torch.nonzero(there)[:, 0]
    zeros = lambda *s: torch.zeros(*s, dtype=torch.float64)
    out = {"loss": zeros(rows), "lse": zeros(rows), "dx": zeros(*x.shape), "d_weight": zeros(*weight.shape)}
    size = {k: v.clone() for k, v in out.items()}
    if len(kept):
        xs, l = x[kept], scale * x[kept] @ weight.t()
        big = (abs(scale) * xs.abs() @ weight.abs().t()).amax(1)
        lse = torch.logsumexp(l, 1)
        at = torch.arange(len(kept))
        out["loss"][kept] = lse - l[at, label[kept].long()] + z_weight * lse ** 2
        out["lse"][kept] = lse
        size["loss"][kept], size["lse"][kept] = big * (2 + 2 * z_weight * lse.abs()), big
        use = lse if lse_given is None else lse_given[kept]
        p = torch.exp(l - use[:, None])
        g = p * (1 + 2 * z_weight * use[:, None])
        g[at, label[kept].long()] -= 1
        f = (w[kept] * d_total * scale)[:, None]
        out["dx"][kept], out["d_weight"] = f * (g @ weight), (f * g).t() @ xs
        most = g.abs() + p * (1 + 2 * z_weight * use[:, None].abs())
        size["dx"][kept], size["d_weight"] = f.abs() * (most @ weight.abs()), (f.abs() * most).t() @ xs.abs()
        size["big"] = big
    out["total"] = (w[kept] * out["loss"][kept]).sum().reshape(1)
    size["total"] = (w[kept].abs() * (size["loss"][kept] + out["loss"][kept].abs())).sum().reshape(1)
    return out, size
