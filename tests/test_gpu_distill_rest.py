"""What a teacher that is sure of an id leaves to the ids that its list leaves out (DOMINO_DISTILL_TAIL): the rest, 1 - sum q,
has to be good to its own size for the loss and the gradient of the others to be.

Bounds, t <= 32 base-2 octaves below the row's greatest.  log p_b: three roundings of half an ulp(16 .. 32), 1.5 * 2^-19 ln 2 =
2e-6; exponentials (2^-22 each, three of them for 16-bit logits: the term, the factor of its unit, the listed id's) and the
quotient 8e-7: D = 2.8e-6.  The rest: -expm1 of the greatest score and the sum of the other q, each within 2^-22 of values of
1 - q_max at most: 2^-21 (1 - q_max).  The loss's derivative by log p_b is p_b - q_b, by q_b and the rest log(q_b / p_b):
  |error of the loss| <= D sum_b |p_b - q_b| + 2^-21 (1 - q_max) |log(rest / p_rest)| + 2^-21 sum_b q_b |log(q_b / p_b)|,
the last for the rounding of q_b (2^-22) and of the terms.  An unlisted id's gradient is (g w / T) p_v / p_rest (p_rest - rest):
  |error| <= (g w / T) (p_v / p_rest) (2 D p_rest + D rest + 2^-21 (1 - q_max)) + eps / 2 |dx_v|;
the gradient alone adds the rounding of two stored logarithms below 32 (2^-20 each, half an ulp) to every p_v and p_rest: 2 D
covers them once more."""
import math

import numpy as np
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import rows_reference as ref
from tests.test_gpu_distill import TAIL, run
from tests.test_gpu_sample_filtered import DEV, TYPES, logits

pytestmark = pytest.mark.gpu

F32, BF16, F16 = b.DOMINO_F32, b.DOMINO_BF16, b.DOMINO_F16
D = 2.8e-6


def parts(x, ids, scores, T):
    """Of one row in 64 bits: (loss, its bound, q, rest, p of every id, p_rest, unlisted ids)."""
    z = x.astype(np.float64) / float(np.float32(T))
    ok, q, rest = ref.teacher(ids, scores, z.size, T, True)
    out = np.ones(z.size, bool)
    out[ids[ok]] = False
    p = np.exp(z - ref.lse(z))
    p_rest = math.exp(ref.lse(z[out]) - ref.lse(z))
    i, q = ids[ok], q[ok]
    last = abs(math.log(rest / p_rest))
    tol = D * (np.abs(p[i] - q).sum() + abs(p_rest - rest)) + 2.0 ** -21 * ((1 - q.max()) * last + (q * np.abs(np.log(q / p[i]))).sum()
                                                                              + rest * last)
    return ref.distill(x, ids, scores, T, True)[0], tol, q, rest, p, p_rest, out


@pytest.mark.parametrize("sure", [7.0, 12.0, 16.0, 19.0])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_a_teacher_that_is_sure_of_an_id(dtype, sure):
    """One logit lies `sure` above the sum of the others, about: the rest is e^-7 to e^-19 of the mass."""
    rows, V, kt = 4, 5000, 8
    x = logits(rows, V, dtype, 81, std=1.0)
    x[:, 77] = torch.logsumexp(x.float(), 1).to(x.dtype) + sure
    g = torch.Generator().manual_seed(82)
    t = x.double().cpu() + 0.3 * torch.randn((rows, V), generator=g).double()
    v, i = torch.topk(t, kt, dim=1)
    ids, scores = i.int(), (v - torch.logsumexp(t, 1, keepdim=True)).float()
    xs, eps = x.double().cpu().numpy(), torch.finfo(TYPES[dtype]).eps / 2
    up = torch.full((rows,), 1024.0)
    loss, lse, _ = run("loss", x, dtype, ids, scores, 1.0, TAIL)
    both, _, dx = run("both", x, dtype, ids, scores, 1.0, TAIL, up=up)
    _, _, alone = run("grad", x, dtype, ids, scores, 1.0, TAIL, up=up, lse=lse)
    for r in range(rows):
        e, tol, q, rest, p, p_rest, out = parts(xs[r], ids[r].numpy(), scores[r].numpy(), 1.0)
        for got in (loss, both):
            assert abs(got[r] - e) <= tol, (r, got[r], e, tol)
        want = 1024.0 * p[out] / p_rest * (p_rest - rest)
        slack = 1024.0 * p[out] / p_rest * (2 * D * p_rest + D * rest + 2.0 ** -21 * (1 - q.max()))
        tiny = torch.finfo(TYPES[dtype]).smallest_normal * eps
        for d, times in ((dx, 1.0), (alone, 2.0)):
            off = np.abs(d[r].double().cpu().numpy()[out] - want)
            assert (off <= times * slack + eps * np.abs(want) + tiny).all(), (r, (off - eps * np.abs(want) - times * slack).max(), rest)
