"""The log-probability of a draw that is nearly certain (domino_sample_filtered): it is near 0, and good to its own size.

Bound.  logp = -log1p(o / w), o what the others weigh and w the token's.  The others' weights are fp32 below 2^-11 of the
greatest, 2^-19 of their value (tests/test_gpu_sample_filtered.py), exact sums; o and w round to fp32 (2^-24 each), the quotient
too, log1p is good to 2^-23: |error| <= (2^-19 + 2^-21) |logp| < 2^-18 |logp|, plus V 2^-44 of weights that are rounded to
nothing or up."""
import numpy as np
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import rows_reference as ref
from tests.test_gpu_sample_filtered import DEV, logits, run

pytestmark = pytest.mark.gpu

F32, BF16, F16 = b.DOMINO_F32, b.DOMINO_BF16, b.DOMINO_F16
RULES = {"none": {}, "topk": dict(k=[2, 50, 400, 1000]), "minp": dict(m=[1e-3, 1e-6, 1e-7, 1e-9]),
         "topk-topp": dict(k=[50] * 4, p=[0.9999999] * 4), "topp": dict(p=[0.9999999] * 4)}


@pytest.mark.parametrize("rule", sorted(RULES))
@pytest.mark.parametrize("dtype,V", [(F32, 700), (BF16, 5001), (F32, 151936), (F16, 151935)])
def test_the_log_probability_of_a_sure_draw(dtype, V, rule):
    x = logits(4, V, dtype, 91, std=1.0)
    for r, sure in enumerate((2.0, 4.0, 7.0, 10.0)):
        x[r, V // 3] = (torch.logsumexp(x[r].float(), 0) + sure).to(x.dtype)
    u = torch.full((4,), 0.5)
    got, lp = run(x, dtype, u, **RULES[rule])
    xs = x.double().cpu().numpy()
    for r in range(4):
        a = {n: float(np.float32(v[r])) if n != "k" else v[r] for n, v in RULES[rule].items()}
        e, elp, margin = ref.draw(xs[r], 0.5, **a)
        assert got[r] == e == V // 3
        if margin > 1e-7:  # (which ids top-p keeps is not in doubt)
            assert abs(lp[r] - elp) <= 2.0 ** -18 * abs(elp) + V * 2.0 ** -44, (r, lp[r], elp)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_only_kept_id_has_log_probability_0(dtype):
    x = logits(4, 3000, dtype, 92)
    for a in (dict(k=[1] * 4), dict(p=[0.0] * 4), dict(T=[0.0] * 4)):
        _, lp = run(x, dtype, torch.full((4,), 0.5), **a)
        assert (lp == 0).all()
    # min_p = 1 keeps every id that has the greatest probability (two in a row of bf16 logits): log(1 / n)
    n = (x == x.amax(1, keepdim=True)).sum(1).cpu().numpy()
    _, lp = run(x, dtype, torch.full((4,), 0.5), m=[1.0] * 4)
    assert (np.abs(lp + np.log(n)) <= 2.0 ** -23).all() and (lp[n == 1] == 0).all() and (n == 1).any()
    x[:, 5] = float("inf")
    _, lp = run(x, dtype, torch.full((4,), 0.5, device=DEV).cpu())
    assert (lp == 0).all()
