"""The oracle of the head's losses against torch's own cross entropy and divergence in float64, against differences, and
against sums written out."""
import math

import pytest
import torch

from oracle import head_oracle as orc

F64 = torch.float64


def small(seed, t=5, v=11, d=6):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(t, d, generator=g, dtype=F64), torch.randn(v, d, generator=g, dtype=F64), g


@pytest.mark.parametrize("softcap,temperature,z_loss", [(0.0, 1.0, 0.0), (3.0, 1.0, 0.0), (0.0, 2.0, 0.1), (2.0, 0.5, 0.3)])
def test_cross_entropy_is_torchs_and_its_gradient_autograds(softcap, temperature, z_loss):
    x, w, g = small(1)
    labels = torch.tensor([3, -100, 0, 10, 11])
    weights = torch.tensor([0.5, 2.0, 1.5, -0.25, 9.0], dtype=F64)
    x.requires_grad_(True)
    z = x @ w.T * 1.3
    if softcap:
        z = softcap * torch.tanh(z / softcap)
    z = z / temperature
    y = torch.where(labels < 11, labels, torch.full_like(labels, -100))
    each = torch.nn.functional.cross_entropy(z, y, ignore_index=-100, reduction="none")
    each = each + torch.where(y >= 0, z_loss * torch.logsumexp(z, 1) ** 2, torch.zeros(5, dtype=F64))
    kept = torch.where(y >= 0, weights, torch.zeros(5, dtype=F64))
    ((kept * each).sum() / kept.sum()).backward()
    o = orc.head(x.detach(), w, *orc.label_rows(labels, 11), scale=1.3, softcap=softcap, temperature=temperature,
                 z_loss=z_loss, weights=weights)
    assert torch.allclose(o["loss"], each.detach(), atol=1e-13)
    assert torch.allclose(o["d_x"], x.grad, atol=1e-13)
    assert torch.allclose(o["totals"], torch.stack([(kept * each.detach()).sum(), kept.sum()]), atol=1e-13)
    assert (o["d_x"][1] == 0).all() and o["lse"][4] == 0


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("softcap", [0.0, 2.5])
def test_distillation_gradient_against_differences(tail, softcap):
    x, w, g = small(2)
    u = torch.randn(5, 11, generator=g, dtype=F64)
    index = torch.stack([torch.randperm(11, generator=g)[:4] for _ in range(5)])
    index[1, 2:] = -1
    index[3] = torch.tensor([7, 7, 2, 40])
    logit = torch.gather(u, 1, index.clamp(0, 10))
    lse = torch.logsumexp(u / 1.7, 1) + 0.2 if tail else None
    args = dict(softcap=softcap, temperature=1.7, z_loss=0.05)
    rows = orc.teacher(index, logit, 11, 1.7, lse)
    o = orc.head(x, w, *rows, **args)
    h = 1e-6
    for t in range(5):
        for j in range(6):
            up, down = x.clone(), x.clone()
            up[t, j] += h
            down[t, j] -= h
            f = [orc.head(y, w, *rows, gradient=False, **args) for y in (up, down)]
            diff = (f[0]["totals"][0] - f[1]["totals"][0]) / (2 * h) / o["totals"][1]
            assert abs(diff - o["d_x"][t, j]) < 1e-8


def test_divergence_of_the_whole_vocabulary_is_torchs():
    x, w, g = small(3)
    u = torch.randn(5, 11, generator=g, dtype=F64)
    index = torch.arange(11).repeat(5, 1)
    z = x @ w.T / 2
    want = torch.nn.functional.kl_div(torch.log_softmax(z, 1), torch.log_softmax(u / 2, 1), log_target=True,
                                      reduction="none").sum(1)
    for lse in (None, torch.logsumexp(u / 2, 1)):
        o = orc.head(x, w, *orc.teacher(index, u, 11, 2.0, lse), temperature=2.0)
        assert torch.allclose(o["loss"], want, atol=1e-12)


def test_what_the_list_leaves_over_is_one_class():
    x, w, g = small(4, t=1)
    u = torch.randn(1, 11, generator=g, dtype=F64)
    p, q = torch.softmax(x @ w.T, 1)[0], torch.softmax(u, 1)[0]
    index = torch.tensor([[4, 9]])
    o = orc.head(x, w, *orc.teacher(index, u[:, [4, 9]], 11, 1.0, torch.logsumexp(u, 1)))
    r, s = 1 - q[4] - q[9], 1 - p[4] - p[9]
    want = q[4] * math.log(q[4] / p[4]) + q[9] * math.log(q[9] / p[9]) + r * math.log(r / s)
    assert abs(float(o["loss"][0]) - float(want)) < 1e-13


def test_one_entry_of_a_teacher_is_a_label():
    x, w, _ = small(5)
    labels = torch.tensor([3, 0, 10, 5, -1])
    a = orc.head(x, w, *orc.label_rows(labels, 11), z_loss=0.01)
    b = orc.head(x, w, *orc.teacher(labels[:, None], torch.full((5, 1), 7.0), 11), z_loss=0.01)
    for n in ("loss", "lse", "d_x", "totals"):
        assert torch.allclose(a[n], b[n], atol=1e-14)


def test_a_planted_mistake_is_outside_the_bounds():
    x, w, g = small(6)
    labels = torch.tensor([3, 0, 10, 5, 1])
    o = orc.head(x, w, *orc.label_rows(labels, 11))
    wrong = orc.head(x, w, *orc.label_rows((labels + 1) % 11, 11))
    assert ((wrong["d_x"] - o["d_x"]).abs() > o["bound"]["d_x"]).any(1).all()
    assert ((wrong["loss"] - o["loss"]).abs() > o["bound"]["loss"]).all()
