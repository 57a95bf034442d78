"""Sequences that run past the end of their table: the tokens that have a place keep it, the others are turned and
nobody's key is overwritten; attention gives every token what its place sees of the keys that are there."""
import math

import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import paged_reference as ref
from tests.test_gpu_paged_attend import randq, run
from tests.test_gpu_paged_rope import close, randn, speeds

pytestmark = pytest.mark.gpu
DEV = "cuda"
CAUSAL, FULL, TREE = b.DOMINO_MASK_CAUSAL, b.DOMINO_MASK_FULL, b.DOMINO_MASK_TREE

# pages, page, new tokens, tokens past the table
ENDS = [(4, 16, 4, 2), (4, 16, 4, 4), (4, 16, 1, 1), (5, 7, 12, 11), (3, 64, 33, 1), (1, 8, 20, 3),
        (4, 16, 1, 2), (4, 16, 1, 900), (5, 7, 6, 7), (2, 128, 40, 5000)]  # the tokens before these are past it already


def _full(pages, page, n, past, hkv, D, dtype, seed):
    """A sequence whose table is full, whose length is `past` places more; another one behind it, in order."""
    p = ref.Paged([pages * page, 3], [n, 3], hkv, D, dtype, page, seed=seed)
    p.kv_len[0] += past
    return p, pages * page + past - n  # the first new token's place


@pytest.mark.parametrize("dtype", [b.DOMINO_BF16, b.DOMINO_F32])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("pages,page,n,past", ENDS)
def test_append(pages, page, n, past, tree, dtype):
    hq, hkv, D = 4, 2, 64
    p, first = _full(pages, page, n, past, hkv, D, dtype, past)
    depth = torch.tensor(ref.random_trees(2, max(n, 3), 5)[1], dtype=torch.int32, device=DEV) if tree else None
    q, k, v = (randn((p.tokens, h, D), dtype, 6 + i) for i, h in enumerate((hq, hkv, hkv)))
    q_out, freq = torch.empty_like(q), speeds(D)
    k_was, v_was = p.k.clone(), p.v.clone()
    assert b.domino_rope_append(q, q.stride(0), k, k.stride(0), v, v.stride(0), None, depth, max(n, 3) if tree else 0, freq, 1.0,
                                b.DOMINO_ROPE_HALF, D, hq, p.tokens, q_out, q_out.stride(0), p.cache, p.batch,
                                torch.cuda.current_stream()) == 0
    at = [(0, first + i) for i in range(n)] + [(1, i) for i in range(3)]
    pos = [t if not tree or i == 0 else (first if s == 0 else 0) + int(depth[s, i - 1])
           for (s, t), i in zip(at, list(range(n)) + list(range(3)))]
    pos = torch.tensor(pos, device=DEV)
    want, tol = ref.rotate(q, pos, freq, D, b.DOMINO_ROPE_HALF, 1.0)
    close(q_out, want, tol)
    want, tol = ref.rotate(k, pos, freq, D, b.DOMINO_ROPE_HALF, 1.0)
    seen = torch.zeros(p.k.shape[1:3], dtype=torch.bool, device=DEV)
    for r, (s, t) in enumerate(at):
        if not 0 <= t < (pages * page if s == 0 else 3):
            continue
        where = 0, int(p.table[s, t // page]), t % page
        close(p.k[where], want[r], tol[r])
        assert torch.equal(p.v[where], v[r])
        seen[where[1:]] = True
    same = lambda now, was: (now == was) | (now.isnan() & was.isnan())
    assert bool(same(p.k, k_was)[0][~seen].all()) and bool(same(p.v, v_was)[0][~seen].all())


@pytest.mark.parametrize("dtype", [b.DOMINO_BF16, b.DOMINO_F16, b.DOMINO_F32])
@pytest.mark.parametrize("mask", [CAUSAL, FULL, TREE])
@pytest.mark.parametrize("pages,page,n,past", ENDS + [(40, 16, 70, 69), (16, 128, 130, 100)])
def test_attend(pages, page, n, past, mask, dtype):
    """Against the 64-bit form; its tolerances are those of the reference's head, from the keys that are there."""
    hq, hkv, D = 16, 2, 64
    p, first = _full(pages, page, n, past, hkv, D, dtype, past + 1)
    parents = ref.random_trees(2, max(n - 1, 1), 3)[0] if mask == TREE else None
    parent = torch.tensor(parents, dtype=torch.int32, device=DEV) if parents else None
    q = randq(p.tokens, hq, D, dtype, 8)
    out, lse, status = run(p, q, mask, parent, len(parents[0]) if parents else 0)
    assert status == 0
    kv, scale, u = pages * page, D ** -0.5, torch.finfo(q.dtype).eps / 2
    see = ref.visible(mask, n, kv + past, parents[0] if parents else None)[:, :kv].to(DEV)
    tensor = dtype != b.DOMINO_F32
    k, v = p.read(p.k, 0).double(), p.read(p.v, 0).double()
    for h in range(hq):
        x, kh, vh = q[:n, h].double(), k[:, h // 8], v[:, h // 8]
        z = (scale * (x @ kh.T)).masked_fill(~see, -math.inf)
        some = see.any(1)
        l = torch.logsumexp(z, 1)
        w = torch.where(some[:, None], (z - l[:, None]).exp(), 0.0)
        o, A = w @ vh, w @ vh.abs()
        e = 2 * (D + 8) * 2.0 ** -24 * (scale * (x.abs() @ kh.abs().T)).masked_fill(~see, 0.0).amax(1) + 2.0 ** -20
        tol = u * o.abs() + (e[:, None] + (u if tensor else 0.0)) * A
        if dtype == b.DOMINO_F16:
            tol = tol + 2.0 ** -25 * torch.where(some, z.amax(1) - l, 0.0).exp()[:, None] * (see.double() @ vh.abs())
        assert bool(((out[:n, h].double() - o).abs() <= tol).all()), h
        assert bool((lse[:n, h][~some] == -math.inf).all())
        assert bool(((lse[:n, h].double() - l).abs()[some] <= (e / 2 + 2.0 ** -23 * l.abs())[some]).all()), h
