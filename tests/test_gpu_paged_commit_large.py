"""Accepted nodes moved in caches whose layers a block takes hold 2^31 elements and more."""
import pytest
import torch

from paper_2605_29707_gb300 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("layers", [256, 300])
def test_many_wide_layers(layers):
    """One sequence of many has new tokens: an anchor and two nodes, of which the second is accepted.  The tensors begin off
    16-byte boundaries, so a block counts single elements: 2 x 16384 x 256 of them in every layer."""
    heads, D, B = 16384, 256, 1300
    n = layers * 3 * heads * D
    store = [torch.empty(n + 8, dtype=torch.int16, device=DEV).random_() for _ in range(2)]
    k, v = (x[1:1 + n].view(layers, 3, heads, D) for x in store)
    was = [x.clone() for x in (k, v)]
    i32 = dict(dtype=torch.int32, device=DEV)
    table, kv_len, start = torch.zeros((B, 1), **i32), torch.zeros(B, **i32), torch.full((B + 1,), 3, **i32)
    kv_len[0], start[0] = 3, 0
    nodes, count, new_len = torch.full((B, 2), -1, **i32), torch.zeros(B, **i32), torch.full((B,), -7, **i32)
    nodes[0, 0], count[0] = 1, 1
    cache = b.make_cache(k, v, 3 * heads * D, heads * D, D, 1, 3, heads, D, b.DOMINO_BF16)
    batch = b.make_batch(table, 1, 1, kv_len, start, B)
    assert b.domino_cache_commit(cache, batch, layers, 3 * heads * D, nodes, count, 2, new_len, torch.cuda.current_stream()) == 0
    assert new_len.tolist() == [2] + [0] * (B - 1)
    for x, y in zip((k, v), was):
        assert torch.equal(x[:, 0], y[:, 0]) and torch.equal(x[:, 1], y[:, 2]) and torch.equal(x[:, 2], y[:, 2])
