"""The digits of the distillation loss where the student is near the teacher (domino_distill_loss, _loss_grad), against
the plain 64-bit form of tests/rows_reference.py.

Bound.  The loss is sum_b q_b h(p_b / q_b - 1) + sum_b (q_b - p_b) over the listed ids and the rest, and its derivative by
log p_b is p_b - q_b up to what all p share, which cancels: |error| <= D sum_b |p_b - q_b|, D the error of a log p_b beyond
the shared one.  An argument of base-2 size t has three roundings of half a step (difference, factor, product), 1.5 ulp(t)
ln 2; the exponential is good to 2^-22, the quotient by Z adds 2^-23.  The listed ids are the teacher's best and lie within
about 7 / T of the row's maximum: t < 16 / T, so D < 1.4e-6 at T = 1 (ulp(8 .. 16) = 2^-20, halved: half of the listed lie
below t = 8), 8.6e-7 at 2.5, 6.1e-7 at 4.  A teacher that differs by a normal deviate of 1 / T in each logit has
|p_b - q_b| near q_b / T against a term of q_b / (2 T^2): sum |p_b - q_b| is about 2 T times the loss.  That is 2.8e-6,
4.3e-6 and 4.9e-6 of the loss; the rounding of q_b (2^-23, times log(q_b / p_b), near 1 / T) and of the terms' sum are an
order below.  DIGITS = 5e-6.
Where places share an id the loss is no divergence any more: it is one, K = sum_b q_b log(q_b / p_b), plus N = sum_j q_j
log(q_j / q_b) <= 0, and the bound above is K's (its derivation nowhere uses N, and a bucket whose q_b is twice p_b has
|p_b - q_b| = 2.6 of its term, log 2 - 1 / 2, too).  N's terms have the rounding of a quotient (2^-24, in the logarithm of
1 / 2 or less), of the logarithm (2^-23), of q_j (2^-23) and of the product (2^-24): 2^-21 |N|.  A row of such a list is
held to DIGITS K + 2^-21 |N|, K = loss - N."""
import numpy as np
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import rows_reference as ref
from tests.test_gpu_distill import RENORM, TAIL, lists, run
from tests.test_gpu_sample_filtered import TYPES, logits

pytestmark = pytest.mark.gpu

F32, BF16, F16 = b.DOMINO_F32, b.DOMINO_BF16, b.DOMINO_F16
DIGITS = 5e-6


def bound(want, ids, scores, V, T, tail):
    """DIGITS K + 2^-21 |N| of one row; N is 0 where no id is shared."""
    ok, q, _ = ref.teacher(ids, scores, V, T, tail)
    total = np.zeros(V)
    np.add.at(total, ids[ok], q[ok])
    n = sum(a * np.log(a / total[i]) for a, i in zip(q[ok], ids[ok]) if a > 0)
    return DIGITS * (want - n) + 2.0 ** -21 * abs(n)


@pytest.mark.parametrize("mode", [TAIL, RENORM])
@pytest.mark.parametrize("T", [1.0, 2.5, 4.0])
@pytest.mark.parametrize("V,kt,dtype", [(40000, 8, F32), (40000, 64, BF16), (151936, 8, BF16), (151936, 64, F32), (151936, 8, F16)])
def test_the_loss_is_right_to_its_own_size(V, kt, dtype, T, mode):
    rows = 6
    x = logits(rows, V, dtype, 40 + kt, std=5.1)
    ids, scores = lists(x, kt, mode, T, 40 + V % 7)
    xs = x.double().cpu().numpy()
    want = np.array([ref.distill(xs[r], ids[r].numpy(), scores[r].numpy(), T, mode == TAIL)[0] for r in range(rows)])
    tol = np.array([bound(want[r], ids[r].numpy(), scores[r].numpy(), V, T, mode == TAIL) for r in range(rows)])
    assert (tol <= 1.01 * DIGITS * want).sum() >= rows - 1
    for part in ("loss", "both"):
        loss, _, _ = run(part, x, dtype, ids, scores, T, mode)
        assert (np.abs(loss - want) <= tol).all(), (part, loss / want - 1, tol / want)


@pytest.mark.parametrize("T", [1.0, 3.0])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_a_student_that_is_the_teacher_loses_nothing(dtype, T):
    """The teacher's list holds the student's own log-probabilities: every p_b / q_b is 1 to 1e-5 (the rest, at least a
    hundredth, is a difference of numbers near 1), so 0 <= loss <= (1e-5)^2."""
    V, kt, rows = 60000, 16, 4
    x = logits(rows, V, dtype, 47, std=4.0)
    z = x.double().cpu() / T
    v, i = torch.topk(z, kt, dim=1)
    scores = (v - torch.logsumexp(z, 1, keepdim=True)).float()
    assert (scores.double().exp().sum(1) < 0.99).all()
    loss, _, _ = run("loss", x, dtype, i.int(), scores, T, TAIL)
    assert (loss >= 0).all() and (loss <= 1e-10).all(), loss


@pytest.mark.parametrize("mode", [TAIL, RENORM])
def test_an_id_in_several_places(mode):
    """Three places share an id: their own division of its mass counts, sum_j q_j log(q_j / p)."""
    V, T = 500, 2.0
    x = logits(3, V, F32, 48, std=1.0)
    ids = torch.tensor([[7, 9, 7, 7], [7, 7, -1, 9], [3, 4, 5, 6]]).int()
    scores = torch.log(torch.tensor([[0.2, 0.3, 0.1, 0.05], [0.25, 0.25, 0.9, 0.1], [0.2, 0.1, 0.3, 0.1]]))
    xs = x.double().cpu().numpy()
    for part in ("loss", "both"):
        loss, _, _ = run(part, x, F32, ids, scores, T, mode)
        for r in range(3):
            want = ref.distill(xs[r], ids[r].numpy(), scores[r].numpy(), T, mode == TAIL)[0]
            assert abs(loss[r] - want) <= bound(want, ids[r].numpy(), scores[r].numpy(), V, T, mode == TAIL), (r, loss[r], want)
