"""The gradient alone (domino_distill_grad) on rows whose log-sum-exps lie so far from zero that fp32 does not tell the
logits of such a row apart by them: every unlisted id masked with a finite value, rows with a large common offset.  Bounds
as in tests/test_gpu_distill_masks.py; the two entry points agree within twice that."""
import numpy as np
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests.test_gpu_distill import RENORM, TAIL, run
from tests.test_gpu_distill_masks import hold, lists, only_listed
from tests.test_gpu_sample_filtered import TYPES, logits

pytestmark = pytest.mark.gpu

F32, BF16, F16 = b.DOMINO_F32, b.DOMINO_BF16, b.DOMINO_F16
LOW = "lowest"


def both_agree(x, dtype, ids, scores, T, mode, up=None):
    scale = 1.0 if up is None else float(up[0])
    loss, lse, dx = run("both", x, dtype, ids, scores, T, mode, up=up)
    _, _, alone = run("grad", x, dtype, ids, scores, T, mode, up=up, lse=lse)
    hold(x, dtype, ids, scores, T, mode, loss, dx, scale)
    hold(x, dtype, ids, scores, T, mode, None, alone, scale)
    _, _, skewed = run("grad", x, dtype, ids, scores, T, mode, up=up, pad=3, skew=1, lse=lse)
    assert torch.equal(alone, skewed)
    y = x.clone()
    _, _, placed = run("grad", y, dtype, ids, scores, T, mode, up=up, lse=lse, inplace=True)
    assert placed.data_ptr() == y.data_ptr() and torch.equal(placed, alone)


@pytest.mark.parametrize("mode", [RENORM, TAIL])
@pytest.mark.parametrize("T", [1.0, 1.3, 1.5, 3.0])
@pytest.mark.parametrize("dtype,value,V", [(F32, LOW, 3000), (F32, -1e10, 40001), (F32, -3e5, 3000), (F32, -1e20, 700), (BF16, LOW, 40000),
                                           (BF16, -1e10, 3001), (BF16, -1e5, 3000), (F16, LOW, 17001), (F16, -2e4, 3000)])
def test_nothing_but_listed_ids(dtype, value, V, T, mode):
    x = logits(3, V, dtype, 71)
    ids, scores = only_listed(x, torch.finfo(TYPES[dtype]).min if value == LOW else value, mode)
    both_agree(x, dtype, ids, scores, T, mode, torch.full((3,), 4.0))


@pytest.mark.parametrize("mode", [RENORM, TAIL])
def test_masks_of_several_depths(mode):
    """Of the unlisted ids a few are masked less deeply than the others: they alone have the rest's gradient."""
    x = logits(3, 20000, F32, 72)
    ids, scores = only_listed(x, -1e10, mode)
    few = torch.arange(0, 20000, 997)
    few = few[~torch.isin(few, ids.long())]
    x[:, few] = -0.9e10
    both_agree(x, F32, ids, scores, 1.3, mode)


@pytest.mark.parametrize("mode", [RENORM, TAIL])
@pytest.mark.parametrize("shift", [-4000.0, 4000.0, 60000.0])
def test_rows_with_a_common_offset(shift, mode):
    x = logits(3, 33000, F32, 73) + shift
    ids, scores = lists(x, torch.ones(x.shape, dtype=torch.bool), mode, 1.3, 74)
    both_agree(x, F32, ids, scores, 1.3, mode)


def test_a_weight_of_zero_and_an_empty_list_there():
    x = logits(3, 3000, F32, 75)
    ids, scores = only_listed(x, -1e10, TAIL)
    ids[1] = -1
    w = torch.tensor([0.0, 1.0, 1.0])
    loss, lse, dx = run("both", x, F32, ids, scores, 1.3, TAIL, w)
    _, _, alone = run("grad", x, F32, ids, scores, 1.3, TAIL, w, lse=lse)
    assert (alone[0] == 0).all() and (dx[0] == 0).all() and loss[0] == 0
    assert alone[1].abs().max() <= 1e-6 and np.isfinite(alone.cpu().numpy()).all()
