"""The plain 64-bit forms that the GPU's row operators are held to, against cases worked by hand (CPU)."""
import numpy as np

from tests import rows_reference as ref


def test_draw_by_hand():
    """Probabilities 0.4, 0.1, 0.3, 0.2: each filter's kept ids and the draw in id order."""
    x = np.log(np.array([0.4, 0.1, 0.3, 0.2]))
    assert ref.kept_ids(x)[0].tolist() == [0, 1, 2, 3]
    assert ref.kept_ids(x, k=2)[0].tolist() == [0, 2]
    assert ref.kept_ids(x, p=0.69)[0].tolist() == [0, 2]        # 0.4 lies before id 2, 0.7 before id 3
    assert ref.kept_ids(x, p=0.71)[0].tolist() == [0, 2, 3]
    assert ref.kept_ids(x, k=2, p=0.5)[0].tolist() == [0]       # 0.4 / 0.7 of the two lies before id 2
    assert ref.kept_ids(x, m=0.6)[0].tolist() == [0, 2]
    assert ref.kept_ids(x, T=0.0)[0].tolist() == [0]
    assert ref.kept_ids(x, p=0.0)[0].tolist() == [0]
    t, lp, _ = ref.draw(x, 0.45)
    assert t == 1 and abs(lp - np.log(0.1)) < 1e-12
    t, lp, _ = ref.draw(x, 0.6, k=2)
    assert t == 2 and abs(lp - np.log(0.3 / 0.7)) < 1e-12
    t, lp, _ = ref.draw(x, 0.3, T=0.5)                          # squared: 0.16, 0.01, 0.09, 0.04 of 0.3
    assert t == 0 and abs(lp - np.log(0.16 / 0.3)) < 1e-12


def test_ties_go_to_the_lower_id():
    x = np.array([1.0, 2.0, 2.0, 2.0, 0.0])
    assert ref.kept_ids(x, k=2)[0].tolist() == [1, 2]
    assert ref.draw(x, 0.5, T=-1.0)[0] == 1
    assert ref.draw(np.array([-0.0, 0.0]), 0.9, T=0.0)[0] == 0


def test_masked_rows():
    x = np.array([-np.inf, 3.0, np.nan, 1.0])
    assert ref.draw(x, 0.999)[0] == 3 and ref.draw(x, 0.0)[0] == 1
    assert ref.draw(np.full(3, -np.inf), 0.5) == (0, -np.inf, 1.0)
    assert ref.draw(np.array([1.0, np.inf, np.inf]), 0.6)[0] == 2


def test_distill_by_hand():
    """Student 1/2, 1/4, 1/4; teacher 3/4 on id 1, and 1/4 on id 2 (renormalised) or left to the rest."""
    x = np.log(np.array([0.5, 0.25, 0.25]))
    ids, q = np.array([1, 2]), np.log(np.array([0.75, 0.25]))
    loss, z, r, g = ref.distill(x, ids, q)
    assert abs(loss - 0.75 * np.log(3.0)) < 1e-12 and abs(z) < 1e-12 and abs(r - np.log(0.5)) < 1e-12
    np.testing.assert_allclose(g, [0.5, -0.5, 0.0], atol=1e-12)
    loss, _, r, g = ref.distill(x, ids[:1], q[:1], tail=True)
    assert abs(r - np.log(0.75)) < 1e-12
    assert abs(loss - (0.75 * np.log(3.0) + 0.25 * np.log(0.25 / 0.75))) < 1e-12
    np.testing.assert_allclose(g, [0.5 - 0.25 * 0.5 / 0.75, -0.5, 0.25 - 0.25 * 0.25 / 0.75], atol=1e-12)


def test_distill_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(3)
    x = rng.normal(size=12)
    ids, s = np.array([4, 7, -1, 4]), np.log(np.array([0.3, 0.2, 0.5, 0.1]))
    for tail in (False, True):
        g = ref.distill(x, ids, s, T=1.7, tail=tail, weight=0.6, up=2.0)[3]
        for v in range(12):
            h = np.zeros(12)
            h[v] = 1e-5
            d = ref.distill(x + h, ids, s, 1.7, tail, 0.6)[0] - ref.distill(x - h, ids, s, 1.7, tail, 0.6)[0]
            assert abs(2.0 * d / 2e-5 - g[v]) < 1e-8
