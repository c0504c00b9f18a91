"""The 64-bit forms of the training-step operators against torch's own derivatives, and against hand-evaluated cases."""
import math

import pytest
import torch

from oracle import training


@pytest.mark.parametrize("post", ["rms", "layer", "none"])
@pytest.mark.parametrize("pre", ["rms", "layer"])
def test_norm_gradients(post, pre):
    torch.manual_seed(0)
    x, y = (torch.randn(5, 7).double().requires_grad_() for _ in range(2))
    vec = {k: torch.randn(7).double().requires_grad_() for k in ("post_weight", "post_bias", "pre_weight", "pre_bias")
           if not (post == "none" and "post" in k)}
    vec["gate"] = torch.randn(3, 7).double().requires_grad_()
    out, _ = training.norm_forward(x, y, post, pre, vec, 2, 0.7, 1e-6, 1e-6)
    a, b = torch.randn(5, 7).double(), torch.randn(5, 7).double()
    grads = torch.autograd.grad((a * out["x_out"]).sum() + (b * out["u"]).sum(), [x, y] + list(vec.values()))
    back, _ = training.norm_backward(out["x_out"], y, out["stats"], a, b, post, pre, vec, 2, 0.7)
    for name, g in zip(["dx", "dy"] + list(vec), grads):
        assert torch.allclose(back[name].reshape(g.shape), g), name


def test_norm_by_hand():
    x = torch.tensor([[3.0, -3.0]]).double()
    out, _ = training.norm_forward(x, None, "none", "rms", {}, 0, 2.0, 0.0, 0.0)
    assert out["x_out"].tolist() == [[6.0, -6.0]] and out["u"].tolist() == [[1.0, -1.0]]
    out, _ = training.norm_forward(x, torch.tensor([[2.0, 6.0]]).double(), "layer", "none", {"gate": torch.tensor([[0.5, 2.0]]).double()}, 0, 1.0, 0.0, 0.0)
    assert out["x_out"].tolist() == [[2.5, -1.0]]


@pytest.mark.parametrize("renormalise", [False, True])
def test_route_gradient(renormalise):
    torch.manual_seed(1)
    l = torch.randn(9, 6).double().requires_grad_()
    d_loss, d_weight = torch.tensor([0.3, 0.2]).double(), torch.randn(9, 3).double()
    r = training.route(l.detach(), None, 3, renormalise, 4, d_loss, d_weight)
    p, lse = torch.softmax(l, 1), torch.logsumexp(l, 1)
    w = p.gather(1, r["expert"])
    w = w / w.sum(1, keepdim=True) if renormalise else w
    balance = 0.0
    for g, part in enumerate(torch.split(p, 4)):
        balance = balance + 6 / (3 * len(part) ** 2) * (r["counts"][g] * part.sum(0)).sum() / 3
    assert torch.allclose(r["loss"], torch.stack((balance, (lse ** 2).mean())))
    assert torch.allclose(r["weight"], w) and torch.equal(r["expert"], torch.topk(l, 3, 1).indices)
    grad, = torch.autograd.grad(d_loss[0] * balance + d_loss[1] * (lse ** 2).mean() + (d_weight * w).sum(), l)
    assert torch.allclose(r["d_logits"], grad)


def test_route_by_hand():
    """Two tokens that agree on one of four experts, every logit alike otherwise: balance is E f P of that expert and of the rest."""
    l = torch.tensor([[math.log(3.0), 0, 0, 0]] * 2, dtype=torch.float64)
    r = training.route(l, None, 1, False, 0)
    assert r["expert"].tolist() == [[0], [0]] and r["counts"].tolist() == [[2, 0, 0, 0]]
    assert abs(float(r["loss"][0]) - 4 * 1.0 * 0.5) < 1e-12 and abs(float(r["loss"][1]) - math.log(6.0) ** 2) < 1e-12
    r = training.route(l, torch.tensor([0, 0]), 2, True, 0)
    assert r["loss"].tolist() == [0.0, 0.0] and r["expert"].tolist() == [[-1, -1]] * 2


def test_distill_gradient():
    torch.manual_seed(2)
    s = torch.randn(4, 11).double().requires_grad_()
    tl, ti = torch.randn(4, 3).double(), torch.tensor([[1, 2, 3], [1, 1, 4], [-1, 2, 20], [-1, -1, -1]])
    label, w, tau = torch.tensor([3, 0, -1, 5]), torch.tensor([1.0, 0.5, 2.0, 1.0]).double(), 1.7
    out = training.distill(s.detach(), tl, ti, label, w, tau, 0.6, 0.4, 0.9)
    total = 0.0
    for r in range(4):
        kept = (ti[r] >= 0) & (ti[r] < 11)
        if kept.any():
            q = torch.softmax(tl[r][kept] / tau, 0)
            total = total + w[r] * 0.6 * tau ** 2 * (q * (q.log() - torch.log_softmax(s[r] / tau, 0)[ti[r][kept]])).sum()
        if 0 <= label[r] < 11:
            total = total - w[r] * 0.4 * torch.log_softmax(s[r], 0)[label[r]]
    assert torch.allclose(total, out["total"])
    assert torch.allclose(torch.autograd.grad(0.9 * total, s)[0], out["d_student"])
