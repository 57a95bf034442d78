"""Distillation on rows whose masked places hold finite values, low but not the type's lowest: 16-bit logits.

Bounds: what counts in a sum lies within 2^30 of its greatest, an argument of at most 30 with three roundings of half an
ulp(16 .. 32): 1.5 * 2^-19 ln 2 = 2e-6; the exponential's 2^-22, sums of thousands of terms of independent roundings, a
quotient: 3e-6 of a p_v or a p_v / p_rest.  The gradient alone goes by stored logarithms of at most 64 (2^-19, half an ulp) and
by logits / T of the same size (2^-19): 4e-6 more.  |error| <= (g w / T) 1e-5 (p_v + rest p_v / p_rest + q_v) + eps / 2 |dx_v|
+ half the type's smallest subnormal; the loss, 1e-5 (1 + |loss|).
With a tail the rest is 1 - sum q, where that is far below 1 not good to 1e-5 of itself: an exponential of two ulp (2^-22
of a q, and so of their sum, 1 at most) and KT / 2 roundings of sums near 1 (4 * 2^-24 = 2^-22) leave it off by 2^-21, which
an unlisted id has its share of: 2^-21 (g w / T) p_v / p_rest more."""
import math

import numpy as np
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import rows_reference as ref
from tests.test_gpu_distill import RENORM, TAIL, run
from tests.test_gpu_distill_rest import parts
from tests.test_gpu_sample_filtered import DEV, TYPES, logits

pytestmark = pytest.mark.gpu

F32, BF16, F16 = b.DOMINO_F32, b.DOMINO_BF16, b.DOMINO_F16
KT = 8


def exact(x, ids, scores, T, tail, scale):
    """(loss, gradient, the gradient's bound before it is rounded to its type) of one row in 64 bits; shares of the rest relative to its own maximum."""
    z, T = x.astype(np.float64) / float(np.float32(T)), float(np.float32(T))
    ok, q, rest = ref.teacher(ids, scores, z.size, T, tail)
    out = np.ones(z.size, bool)
    out[ids[ok]] = False
    p = np.exp(z - ref.lse(z))
    share = np.zeros(z.size)
    share[out] = np.exp(z[out] - z[out].max())
    share /= share.sum()
    qv = np.zeros(z.size)
    np.add.at(qv, ids[ok], q[ok])
    loss = ref.distill(x, ids, scores, T, tail)[0]
    off = 1e-5 * (p + rest * share + qv) + (2.0 ** -21 * share if tail else 0.0)
    return loss, scale / T * (p - qv - rest * share), abs(scale) / T * off


def hold(x, dtype, ids, scores, T, mode, loss=None, dx=None, scale=1.0):
    xs, eps, tiny = x.double().cpu().numpy(), torch.finfo(TYPES[dtype]).eps / 2, torch.finfo(TYPES[dtype]).smallest_normal
    for r in range(x.shape[0]):
        e, g, size = exact(xs[r], ids[r].numpy(), scores[r].numpy(), T, mode == TAIL, scale)
        if loss is not None:
            assert abs(loss[r] - e) <= 1e-5 * (1 + abs(e)), (r, loss[r], e)
        if dx is not None:
            off = np.abs(dx[r].double().cpu().numpy() - g)
            bad = np.flatnonzero(~(off <= size + eps * np.abs(g) + tiny * eps))
            assert bad.size == 0, (r, bad.size, bad[:4], dx[r][torch.tensor(bad[:4])], g[bad[:4]])


def lists(x, real, mode, T, seed):
    """The teacher keeps to the real ids: its best KT of them."""
    g = torch.Generator().manual_seed(seed)
    t = x.double().cpu() + torch.randn(x.shape, generator=g).double()
    t = torch.where(real, t, torch.tensor(-math.inf).double())
    t = t / T if mode == TAIL else t
    v, i = torch.topk(t, KT, dim=1)
    return i.int(), (v - torch.logsumexp(t, 1, keepdim=True)).float()


def only_listed(x, value, mode):
    """Rows whose every unlisted id is masked, and a teacher that leaves 0.2 to them."""
    rows, V = x.shape
    ids = torch.stack([torch.randperm(V, generator=torch.Generator().manual_seed(r))[:KT] for r in range(rows)]).int()
    keep = x.gather(1, ids.long().to(DEV))
    x.fill_(value)
    x.scatter_(1, ids.long().to(DEV), keep)
    return ids, torch.full((rows, KT), math.log(0.8 / KT))


@pytest.mark.parametrize("mode", [RENORM, TAIL])
@pytest.mark.parametrize("T", [0.5, 1.0, 1.5, 2.0])
@pytest.mark.parametrize("dtype,value", [(BF16, -1e4), (BF16, -1e9), (BF16, -5e9), (BF16, -1e10), (BF16, -1e12), (BF16, -1e20),
                                         (BF16, -1e29), (F16, -3e4), (F16, -65504.0)])
def test_masked_runs_of_16_bit_logits(dtype, value, T, mode):
    V = 4000
    x = logits(4, V, dtype, 61)
    at = torch.arange(V)
    real = torch.ones((4, V), dtype=torch.bool)
    real[0] = (at >= 1000) & ((at < 1500) | (at >= 2600))   # runs ahead of real ids, whole slices
    real[1] = at // 8 % 3 == 2                              # whole units between real ones
    real[2] = (at >= 2000) & (at % 50 == 3)                 # forty real ids
    x.masked_fill_(~real.to(DEV), value)
    ids, scores = lists(x, real, mode, T, 62)
    loss, lse, _ = run("loss", x, dtype, ids, scores, T, mode)
    hold(x, dtype, ids, scores, T, mode, loss)
    for part in ("grad", "both"):
        _, _, dx = run(part, x, dtype, ids, scores, T, mode, lse=lse if part == "grad" else None)
        hold(x, dtype, ids, scores, T, mode, dx=dx)


@pytest.mark.parametrize("mode", [RENORM, TAIL])
@pytest.mark.parametrize("T", [0.5, 1.0, 1.5, 2.0])
@pytest.mark.parametrize("value", [-1e4, -1e9, -1e10, -1e20, -1e29])
def test_16_bit_rows_with_nothing_but_listed_ids(value, T, mode):
    x = logits(3, 4000, BF16, 63)
    ids, scores = only_listed(x, value, mode)
    loss, _, dx = run("both", x, BF16, ids, scores, T, mode)
    hold(x, BF16, ids, scores, T, mode, loss, dx)


@pytest.mark.parametrize("shift", [300.0, -300.0, 3000.0])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_16_bit_logits_far_from_zero(dtype, shift):
    """A row's common offset changes nothing: the loss is held to the bound of tests/test_gpu_distill_rest.py, which knows
    no offset (at 3000 the steps of bf16 are 16: one or two ids have nearly all the mass)."""
    T, V = 1.0, 40000
    x = logits(4, V, dtype, 64) + shift
    ids, scores = lists(x, torch.ones(x.shape, dtype=torch.bool), TAIL, T, 65)
    xs = x.double().cpu().numpy()
    loss, _, dx = run("both", x, dtype, ids, scores, T, TAIL)
    for r in range(4):
        want, tol = parts(xs[r], ids[r].numpy(), scores[r].numpy(), T)[:2]
        assert abs(loss[r] - want) <= tol, (r, loss[r], want, tol)
    hold(x, dtype, ids, scores, T, TAIL, loss, dx)
