"""Accepted nodes moved in all layers of a paged cache: the same bits as one copy after the other, and nothing else."""
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


def commit(p, nodes, count, N, layers):
    new_len = torch.full((p.B,), -7, dtype=torch.int32, device=DEV)
    nd = torch.full((p.B, max(N, 1)), -1, dtype=torch.int32)
    for i, path in enumerate(nodes):
        nd[i, :len(path)] = torch.tensor(path, dtype=torch.int32)
    nd, ct = nd.to(DEV), torch.tensor(count, dtype=torch.int32, device=DEV)
    assert b.domino_cache_commit(p.cache, p.batch, layers, p.layer_stride, nd if N else None, ct, N, new_len,
                                 torch.cuda.current_stream()) == 0
    return new_len.tolist()


def want(p, nodes, skip=()):
    """The caches after the moves, one after the other."""
    out = []
    for x in (p.k, p.v):
        y = x.clone()
        for i, path in enumerate(nodes):
            if i in skip:
                continue
            first = p.kv[i] - (p.new[i] - 1)
            for j, node in enumerate(path):
                s, d = first + node, first + j
                y[:, int(p.table[i, d // p.page]), d % p.page] = y[:, int(p.table[i, s // p.page]), s % p.page]
        out.append(y)
    return out


def bits(x):
    return x.contiguous().view(torch.int32 if x.element_size() == 4 else torch.int16)


def check(p, nodes, N, layers, skip=()):
    k, v = want(p, nodes, skip)
    lens = commit(p, nodes, [len(x) for x in nodes], N, layers)
    assert torch.equal(bits(p.k), bits(k)) and torch.equal(bits(p.v), bits(v))
    assert lens == [-1 if i in skip else p.kv[i] - max(p.new[i] - 1, 0) + len(nodes[i]) for i in range(p.B)]


@pytest.mark.parametrize("dtype", [b.DOMINO_F32, b.DOMINO_BF16, b.DOMINO_F16])
@pytest.mark.parametrize("order,page,D,pad", [("pth", 16, 128, 0), ("pht", 48, 80, 0), ("thp", 1, 64, 8), ("pth", 7, 65, 1), ("hpt", 5, 3, 0)])
@pytest.mark.parametrize("layers", [1, 5])
def test_commit(dtype, order, page, D, pad, layers):
    N = 32
    p = ref.Paged([200, 33, 50, 40, 77], [33, 33, 33, 33, 20], 3, D, dtype, page, order, pad, layers, seed=page)
    nodes = [[3, 5, 6, 9, 12, 13, 20, 21, 30, 31], [], [0, 1, 2], [0, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12], [18]]
    check(p, nodes, N, layers)


def test_every_node_and_long_lists():
    p = ref.Paged([300, 300], [257, 257], 2, 64, b.DOMINO_BF16, 16, layers=2, seed=1)
    check(p, [list(range(256)), list(range(1, 256))], 256, 2)


def test_no_tree_and_no_new_tokens():
    p = ref.Paged([5, 9], [1, 0], 2, 64, b.DOMINO_BF16, 16, layers=2, seed=2)
    check(p, [[], []], 0, 2)


@pytest.mark.parametrize("nodes,count", [([1, 1], 2), ([2, 1], 2), ([1, 16], 2), ([-1], 1), ([1], -1), ([1], 17), ([1, 3], 1 << 30)])
def test_lists_that_are_none_leave_their_sequence_as_it_is(nodes, count):
    p = ref.Paged([40, 40], [17, 17], 2, 64, b.DOMINO_BF16, 16, layers=3, seed=3)
    k, v = want(p, [[], [2, 4]])
    lens = commit(p, [nodes, [2, 4]], [count, 2], 16, 3)
    assert torch.equal(bits(p.k), bits(k)) and torch.equal(bits(p.v), bits(v))
    assert lens == [-1, 26]


def test_places_without_a_page_leave_their_sequence_as_it_is():
    p = ref.Paged([40, 40, 40], [17, 17, 17], 2, 64, b.DOMINO_BF16, 4, layers=2, seed=4)
    good = p.table.clone()
    p.table[0, 7] = -1       # places 28 .. 31: a source
    p.table[2, 6] = p.pages  # places 24 .. 27: a target
    nodes = [[1, 5, 9], [1, 5, 9], [2, 9]]
    broken, p.table = p.table.clone(), good
    k, v = want(p, nodes, skip=(0, 2))
    p.table = broken
    p.batch = b.make_batch(broken, broken.stride(0), broken.shape[1] - 1, p.kv_len, p.start, 3)
    assert commit(p, nodes, [3, 3, 2], 16, 2) == [-1, 27, -1]
    assert torch.equal(bits(p.k), bits(k)) and torch.equal(bits(p.v), bits(v))


def test_lengths_that_hold_no_tree():
    p = ref.Paged([40, 40], [17, 17], 2, 64, b.DOMINO_BF16, 16, seed=5)
    p.kv_len[0], p.kv_len[1] = 16, 1 << 30
    k, v = p.k.clone(), p.v.clone()
    assert commit(p, [[1], [1]], [1, 1], 16, 1) == [-1, -1]
    assert torch.equal(bits(p.k), bits(k)) and torch.equal(bits(p.v), bits(v))
