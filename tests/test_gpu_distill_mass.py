"""Distillation where the teacher's mass is not 1 (lists without an id or with scores of -inf alone, ids in several places
that add up to more, every id listed with less): the gradient of both entry points against the derivative of the loss in
64 bits (automatic differentiation of its definition) and against differences of the GPU's own losses.

Bounds, V = 48, |z| < 4: a p_v has an argument of three roundings of at most 8 (1.5 ulp(8) ln 2 = 1e-6), the
exponential's 2^-22, a sum of 48 terms and a quotient: below 3e-6 of its value, as an R / Z.  The gradient alone goes by two
stored logarithms of size 8 at most (2^-22) and a product by 1 / T of the same size: 2e-6 more.  |error| <= (g w / T)
(5e-6 (Q p_v + rest p_v / p_rest) + 2^-21 q_v) + eps / 2 |dx_v|."""
import math

import numpy as np
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests.test_gpu_distill import RENORM, TAIL, run
from tests.test_gpu_sample_filtered import DEV, TYPES, logits

pytestmark = pytest.mark.gpu

F32, BF16, F16 = b.DOMINO_F32, b.DOMINO_BF16, b.DOMINO_F16
V, KT, T = 48, 48, 1.3
W, UP = 0.75, -2.0


def _lists():
    """[4, KT] ids and scores: no id; scores of -inf; 0.5 + 0.4 on one id and 0.3 on another; 0.8 spread over every id."""
    ids, scores = torch.full((4, KT), -1, dtype=torch.int32), torch.zeros((4, KT))
    ids[1, :3], scores[1, :3] = torch.tensor([4, 0, 40]).int(), -math.inf
    ids[2, :3], scores[2, :3] = torch.tensor([2, 30, 2]).int(), torch.log(torch.tensor([0.5, 0.3, 0.4]))
    share = torch.rand(V, generator=torch.Generator().manual_seed(3)) + 0.1
    ids[3], scores[3] = torch.randperm(V, generator=torch.Generator().manual_seed(4)).int(), torch.log(0.8 * share / share.sum())
    return ids, scores


def _exact(x, ids, scores, mode):
    """(loss, gradient, bound's terms) of one row, 64 bits."""
    z = x.double().cpu().clone().requires_grad_(True)
    ok = ids >= 0
    i, s = ids[ok].long(), scores[ok].double()
    out = torch.ones(V, dtype=torch.bool)
    out[i] = False
    logp = torch.log_softmax(z / float(np.float32(T)), 0)
    if mode == TAIL:
        q = s.exp()
        rest = max(0.0, 1.0 - float(q.sum())) if out.any() else 0.0
    else:
        some = s.numel() and float(s.max()) > -math.inf
        q, rest = torch.softmax(s / float(np.float32(T)), 0) if some else torch.zeros_like(s), 0.0
    # (terms of q = 0 are 0)
    loss = (torch.special.xlogy(q, q) - q * logp[i]).sum()
    if rest > 0:
        loss = loss + rest * (math.log(rest) - torch.logsumexp(logp[out], 0))
    loss = W * loss
    (UP * loss).backward()
    p = logp.detach().exp().numpy()
    qv = np.zeros(V)
    np.add.at(qv, i.numpy(), q.numpy())
    o = out.numpy()
    size = abs(W * UP) / T * (5e-6 * ((float(q.sum()) + rest) * p + (rest * p / p[o].sum() * o if o.any() else 0)) + 2.0 ** -21 * qv)
    return float(loss), z.grad.numpy(), size


@pytest.mark.parametrize("part", ["grad", "both"])
@pytest.mark.parametrize("mode", [RENORM, TAIL])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_gradient_is_the_loss_derivative_whatever_the_mass(dtype, mode, part):
    x = logits(4, V, dtype, 51, std=1.0)
    ids, scores = _lists()
    w, up = torch.full((4,), W), torch.full((4,), UP)
    loss, lse, dx = run("both", x, dtype, ids, scores, T, mode, w, up)
    if part == "grad":
        loss, lse, _ = run("loss", x, dtype, ids, scores, T, mode, w)
        _, _, dx = run("grad", x, dtype, ids, scores, T, mode, w, up, lse=lse)
    eps = torch.finfo(TYPES[dtype]).eps / 2
    for r in range(4):
        e, g, tol = _exact(x[r], ids[r], scores[r], mode)
        assert abs(loss[r] - e) <= 5e-6 * (1 + abs(e)), (r, loss[r], e)
        off = np.abs(dx[r].double().cpu().numpy() - g)
        assert (off <= tol + eps * np.abs(g) + 2.0 ** -24 * eps).all(), (r, off.max(), g[off.argmax()])
        if mode == RENORM and r < 2:
            assert loss[r] == 0 and (dx[r] == 0).all()


@pytest.mark.parametrize("mode", [RENORM, TAIL])
def test_gradient_is_the_loss_difference_whatever_the_mass(mode):
    """Central differences, step h = 2^-4: h^2 / 6 times the third derivative (at most Q + 1 < 2.5 for T >= 1) plus two
    losses' rounding, 5e-6 (1 + loss) each, over 2 h."""
    h = 2.0 ** -4
    x = logits(4, V, F32, 52, std=1.0)
    ids, scores = _lists()
    _, lse, both = run("both", x, F32, ids, scores, T, mode)
    _, _, alone = run("grad", x, F32, ids, scores, T, mode, lse=lse)
    for r in range(4):
        y = x[r].expand(2 * V, V).clone()
        y[:V] += h * torch.eye(V, device=DEV)
        y[V:] -= h * torch.eye(V, device=DEV)
        loss, _, _ = run("loss", y, F32, ids[r].expand(2 * V, -1).contiguous(), scores[r].expand(2 * V, -1).contiguous(), T, mode)
        quotient = (loss[:V] - loss[V:]) / (2 * h)
        tol = 2.5 * h * h / 6 + 2 * 5e-6 * (1 + np.abs(loss).max()) / (2 * h)
        for dx in (both, alone):
            assert np.abs(quotient - dx[r].double().cpu().numpy()).max() <= tol, r
