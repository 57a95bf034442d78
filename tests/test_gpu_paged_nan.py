"""A NaN that a row sees shows in the row's results, wherever the keys are cut between blocks."""
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import paged_reference as ref
from tests.test_gpu_paged_attend import randq, run

pytestmark = pytest.mark.gpu
DEV = "cuda"
CAUSAL, FULL, TREE = b.DOMINO_MASK_CAUSAL, b.DOMINO_MASK_FULL, b.DOMINO_MASK_TREE
TYPES = [b.DOMINO_BF16, b.DOMINO_F16, b.DOMINO_F32]


def set_keys(p, i, first, last, head, value):
    for t in range(first, last):
        p.k[0, int(p.table[i, t // p.page]), t % p.page, head, 3] = value


def shows(out, lse, rows):
    """rows [tokens, hq]: those that are NaN, all others finite."""
    assert torch.equal(lse.isnan(), rows)
    assert torch.equal(out.isnan().all(2), rows) and torch.equal(out.isnan().any(2), rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads", [(8, 8), (16, 8), (4, 1), (32, 32)])
@pytest.mark.parametrize("kv", [1, 2, 128, 129, 257, 1025, 1100, 4097])
def test_the_newest_key_is_nan(kv, heads, dtype):
    """One decoded token whose own key is NaN for one head: the last tile shows it nothing else."""
    hq, hkv = heads
    p = ref.Paged([kv], [1], hkv, 128, dtype, 16, seed=kv)
    q = randq(1, hq, 128, dtype, 1)
    clean, clean_lse, _ = run(p, q, CAUSAL)
    set_keys(p, 0, kv - 1, kv, 0, float("nan"))
    out, lse, status = run(p, q, CAUSAL)
    assert status == 0
    rows = torch.arange(hq, device=DEV)[None] < hq // hkv
    shows(out, lse, rows)
    assert torch.equal(out[~rows], clean[~rows]) and torch.equal(lse[~rows], clean_lse[~rows])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,heads", [(256, (8, 8)), (256, (16, 4)), (40, (64, 8)), (700, (2, 2))])
def test_queries_of_a_prompt_that_are_nan(n, heads, dtype):
    """A prompt from its first token on; NaN queries among its rows, the first and the last."""
    hq, hkv = heads
    p = ref.Paged([n], [n], hkv, 64, dtype, 16, seed=n)
    q = randq(n, hq, 64, dtype, 2)
    clean, clean_lse, _ = run(p, q, CAUSAL)
    rows = torch.zeros((n, hq), dtype=torch.bool, device=DEV)
    for t, h in ((0, 0), (1, hq - 1), (n // 3, 0), (n // 2, 1), (n - 1, 0)):
        q[t, h, 7], rows[t, h] = float("nan"), True
    out, lse, status = run(p, q, CAUSAL)
    assert status == 0
    shows(out, lse, rows)
    assert torch.equal(out[~rows], clean[~rows]) and torch.equal(lse[~rows], clean_lse[~rows])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mask", [CAUSAL, FULL, TREE])
@pytest.mark.parametrize("kv,n,heads", [(5000, 1, (8, 2)), (30000, 3, (4, 1)), (4000, 17, (16, 1)), (3500, 40, (32, 4))])
def test_nan_queries_over_long_contexts(kv, n, heads, mask, dtype):
    hq, hkv = heads
    p = ref.Paged([kv], [n], hkv, 64, dtype, 16, seed=n)
    parents = ref.random_trees(1, n - 1, n)[0]
    parent = torch.tensor(parents, dtype=torch.int32, device=DEV) if n > 1 else None
    q = randq(n, hq, 64, dtype, 3)
    clean, clean_lse, _ = run(p, q, mask, parent, n - 1)
    rows = torch.zeros((n, hq), dtype=torch.bool, device=DEV)
    rows[n // 2, hq - 1] = True
    q[rows] = float("nan")
    out, lse, status = run(p, q, mask, parent, n - 1)
    assert status == 0
    shows(out, lse, rows)
    assert torch.equal(out[~rows], clean[~rows]) and torch.equal(lse[~rows], clean_lse[~rows])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("first,last", [(0, 700), (900, 1700), (0, 3600), (3500, 3600)])
@pytest.mark.parametrize("n,heads", [(1, (8, 2)), (3, (4, 1)), (33, (16, 2))])
def test_stretches_of_nan_keys(first, last, n, heads, dtype):
    """Hundreds of keys of one head are NaN: parts of the cut see nothing but them."""
    hq, hkv = heads
    p = ref.Paged([3600], [n], hkv, 64, dtype, 16, seed=n)
    q = randq(n, hq, 64, dtype, 4)
    clean, clean_lse, _ = run(p, q, CAUSAL)
    set_keys(p, 0, first, last, hkv - 1, float("nan"))
    out, lse, status = run(p, q, CAUSAL)
    assert status == 0
    sees = torch.arange(n, device=DEV)[:, None] + 3600 - n >= first
    rows = sees & (torch.arange(hq, device=DEV)[None] >= hq - hq // hkv)
    shows(out, lse, rows)
    assert torch.equal(out[~rows], clean[~rows]) and torch.equal(lse[~rows], clean_lse[~rows])
