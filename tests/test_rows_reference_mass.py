"""The plain 64-bit distillation where the teacher's mass is not 1: its gradient is the derivative of its loss (CPU)."""
import numpy as np
import pytest

from tests import rows_reference as ref

EMPTY = (np.array([-1, -1]), np.array([0.0, 0.0]))
NOTHING = (np.array([1, 4]), np.array([-np.inf, -np.inf]))
TWICE = (np.array([2, 0, 2]), np.log(np.array([0.5, 0.3, 0.4])))     # sum q = 1.2
EVERY = (np.arange(6), np.log(np.full(6, 0.8 / 6)))                   # sum q = 0.8, and no other id


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("ids,scores", [EMPTY, NOTHING, TWICE, EVERY])
def test_gradient_is_the_difference_quotient_whatever_the_mass(ids, scores, tail):
    x, T = np.array([0.3, -0.8, 1.1, 0.2, -0.1, 0.6]), 1.4
    g = ref.distill(x, ids, scores, T, tail, 0.7, 2.0)[3]
    for v in range(6):
        h = np.zeros(6)
        h[v] = 1e-5
        d = ref.distill(x + h, ids, scores, T, tail, 0.7)[0] - ref.distill(x - h, ids, scores, T, tail, 0.7)[0]
        assert abs(2.0 * d / 2e-5 - g[v]) < 1e-8


def test_a_list_that_teaches_nothing_by_hand():
    """Renormalised: no loss and no gradient.  With a tail: everything on all ids together, which the student has."""
    x = np.log(np.array([0.5, 0.25, 0.25]))
    for tail in (False, True):
        loss, _, _, g = ref.distill(x, np.array([-1]), np.array([0.0]), tail=tail)
        assert abs(loss) < 1e-12 and np.abs(g).max() < 1e-12
