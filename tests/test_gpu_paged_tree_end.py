"""Tokens behind the end of their sequence's tree see nothing, however long the context before the tree is."""
import math

import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import paged_reference as ref
from tests.test_gpu_paged_attend import check, randq, run

pytestmark = pytest.mark.gpu
DEV = "cuda"
TREE = b.DOMINO_MASK_TREE

# context, new tokens of every sequence, tree nodes, hq, hkv, D
CASES = [
    ([127, 128, 129, 200], [9, 9, 9, 9], 6, 4, 2, 64),            # one tile of queries, the last tokens past the tree
    ([700], [3], 1, 8, 8, 128),                                   # some tokens, many CTAs: joined
    ([700, 256, 1, 2000], [30, 30, 30, 5], 20, 16, 2, 128),       # two tiles of queries, the second past the tree in part
    ([3000, 128], [33, 2], 0, 32, 4, 80),                         # the anchor alone
    ([640, 128], [70, 64], 31, 64, 4, 64),                        # several groups, the last ones past the tree altogether
    ([1500], [130], 100, 8, 1, 128),                              # more tokens than a tree kept as bits
]


def _case(context, new, hkv, D, dtype, seed):
    return ref.Paged([c + n for c, n in zip(context, new)], new, hkv, D, dtype, 16, "pht", seed=seed)


@pytest.mark.parametrize("dtype", [b.DOMINO_BF16, b.DOMINO_F16, b.DOMINO_F32])
@pytest.mark.parametrize("context,new,N,hq,hkv,D", CASES)
def test_tokens_past_the_tree_see_nothing(context, new, N, hq, hkv, D, dtype):
    p = _case(context, new, hkv, D, dtype, N + 1)
    parents = ref.random_trees(p.B, N, N)[0]
    out, lse = check(p, randq(p.tokens, hq, D, dtype, 4), TREE, parents)
    for i in range(p.B):
        past = slice(p.start_host[i] + min(N + 1, new[i]), p.start_host[i + 1])
        assert bool((out[past] == 0).all()) and bool((lse[past] == -math.inf).all())


@pytest.mark.parametrize("dtype", [b.DOMINO_BF16, b.DOMINO_F32])
@pytest.mark.parametrize("context,new,N,hq,hkv,D", CASES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_the_context_holds_does_not_reach_them(context, new, N, hq, hkv, D, dtype, bad):
    """The context's keys and values are not finite in places: rows in the tree show them, those past it stay empty."""
    p = _case(context, new, hkv, D, dtype, N + 2)
    parents = ref.random_trees(p.B, N, N)[0]
    parent = torch.tensor(parents, dtype=torch.int32, device=DEV) if N else None
    q = randq(p.tokens, hq, D, dtype, 5)
    p.k[0, int(p.table[0, 0]), 3, :, 1] = float("nan")
    p.v[0, int(p.table[0, 0]), 5, :, 2] = bad
    out, lse, status = run(p, q, TREE, parent, N)
    assert status == 0
    for i in range(p.B):
        a, end = p.start_host[i], p.start_host[i + 1]
        past = slice(a + min(N + 1, new[i]), end)
        assert bool((out[past] == 0).all()) and bool((lse[past] == -math.inf).all())
        some = lse[a:a + min(N + 1, new[i])]
        assert bool(some.isnan().all()) if i == 0 else bool(some.isfinite().all())
