"""Attention over a paged cache against its fp64 form; whatever no row sees is NaN in these caches."""
import math
import random

import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
CAUSAL, FULL, TREE = b.DOMINO_MASK_CAUSAL, b.DOMINO_MASK_FULL, b.DOMINO_MASK_TREE


def randq(tokens, hq, D, dtype, seed, std=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn((tokens, hq, D), generator=g, device=DEV) * std).to(ref.TORCH[dtype])


def run(p, q, mask, parent=None, N=0, scale=None, rows=None, lse=True):
    """out and lse; rows: the tensors have more rows than the sequences, filled with 7."""
    tokens, hq, D = q.shape
    out = torch.full_like(q, 7.0)
    l = torch.full((tokens, hq), 7.0, device=DEV) if lse else None
    n = b.domino_attend_workspace_bytes(tokens, hq, p.cache)
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)
    s = torch.cuda.current_stream()
    rc = b.domino_attend_paged(q, q.stride(0), tokens, hq, p.cache, p.batch, scale or D ** -0.5, mask, parent, N, out, out.stride(0), l, ws,
                               n, s)
    assert rc == 0
    return out, l, b.domino_check_status(ws, s)


def tensor_path(p, dtype):
    s = p.k.stride()
    return dtype != b.DOMINO_F32 and p.D <= 128 and p.D % 8 == 0 and p.page % 8 == 0 and all(x % 8 == 0 for x in s[1:4])


def check(p, q, mask, parents=None, scale=None):
    N = len(parents[0]) if parents is not None else 0
    parent = torch.tensor(parents, dtype=torch.int32, device=DEV) if N else None
    out, lse, status = run(p, q, mask, parent, N, scale)
    assert status == 0
    want, wl, tol, ltol = ref.attend(p, q, scale or p.D ** -0.5, mask, parents, tensor_path(p, p.dtype))
    n = p.start_host[-1]
    err, lerr = (out[:n].double() - want[:n]).abs(), (lse[:n].double() - wl[:n]).abs()
    empty = wl[:n] == -math.inf
    assert bool((lse[:n][empty] == -math.inf).all()) and bool((out[:n][empty] == 0).all())
    assert bool((err <= tol[:n]).all()), (float((err - tol[:n]).max()), float((err / tol[:n].clamp(min=1e-30)).max()))
    assert bool((lerr <= ltol[:n])[~empty].all()), float((lerr - ltol[:n])[~empty].max())
    assert bool((out[n:] == 7.0).all()) and bool((lse[n:] == 7.0).all())
    return out, lse


SHAPES = [  # kv, new, hq, hkv, D, page, order
    ([1], [1], 4, 4, 128, 16, "pth"),
    ([1000], [1], 16, 8, 128, 16, "pth"),
    ([127, 128, 129, 255, 256, 257], [1] * 6, 8, 2, 128, 16, "pht"),
    ([40, 300, 17, 1025], [1, 17, 0, 5], 12, 4, 64, 48, "pth"),
    ([700, 3, 90], [200, 3, 90], 14, 2, 80, 24, "pht"),
    ([513, 2], [129, 2], 5, 5, 96, 8, "htp"),
    ([600, 1500], [300, 33], 21, 3, 72, 64, "pth"),
    ([333], [65], 128, 1, 128, 256, "pth"),
    ([2300], [2], 3, 1, 8, 128, "pth"),
    ([5000, 4999, 1], [1, 1, 1], 40, 8, 128, 16, "pht"),
    ([450, 131], [9, 4], 65, 1, 64, 200, "pth"),
    ([260, 1000], [150, 40], 6, 2, 104, 136, "pht"),
]


@pytest.mark.parametrize("mask", [CAUSAL, FULL])
@pytest.mark.parametrize("dtype", [b.DOMINO_BF16, b.DOMINO_F16])
@pytest.mark.parametrize("kv,new,hq,hkv,D,page,order", SHAPES)
def test_attend(kv, new, hq, hkv, D, page, order, dtype, mask):
    p = ref.Paged(kv, new, hkv, D, dtype, page, order, seed=sum(kv))
    check(p, randq(p.tokens, hq, D, dtype, 1), mask)


@pytest.mark.parametrize("dtype,kv,new,hq,hkv,D,page,order,pad", [
    (b.DOMINO_F32, [300, 5, 70], [40, 5, 1], 6, 2, 64, 16, "pth", 0),
    (b.DOMINO_F32, [100], [3], 2, 1, 33, 5, "pht", 2),
    (b.DOMINO_BF16, [300, 5, 70], [40, 5, 1], 6, 2, 256, 16, "pth", 0),
    (b.DOMINO_BF16, [130, 9], [9, 9], 4, 2, 64, 1, "pth", 0),
    (b.DOMINO_F16, [130, 9], [9, 9], 4, 2, 60, 16, "pht", 0),
    (b.DOMINO_F16, [130, 9], [9, 9], 4, 2, 64, 16, "pth", 1),
    (b.DOMINO_BF16, [130, 9], [9, 9], 3, 3, 1, 7, "pth", 0),
])
@pytest.mark.parametrize("mask", [CAUSAL, FULL, TREE])
def test_attend_of_other_types_and_layouts(dtype, kv, new, hq, hkv, D, page, order, pad, mask):
    p = ref.Paged(kv, new, hkv, D, dtype, page, order, pad, seed=3)
    parents = ref.random_trees(p.B, 39, 2)[0] if mask == TREE else None
    check(p, randq(p.tokens, hq, D, dtype, 2), mask, parents)


@pytest.mark.parametrize("dtype", [b.DOMINO_BF16, b.DOMINO_F16])
@pytest.mark.parametrize("kv,new,hq,hkv,D,page,N", [
    ([17, 400, 18, 150], [17, 17, 17, 9], 8, 2, 128, 16, 16),
    ([1000, 65, 129], [65, 65, 65], 32, 4, 64, 32, 64),
    ([300, 257], [257, 257], 10, 2, 128, 64, 256),
    ([2049], [33], 64, 8, 128, 32, 32),
    ([64], [5], 7, 1, 80, 48, 4),
])
def test_attend_trees(dtype, kv, new, hq, hkv, D, page, N):
    p = ref.Paged(kv, new, hkv, D, dtype, page, "pht", seed=N)
    check(p, randq(p.tokens, hq, D, dtype, 4), TREE, ref.random_trees(p.B, N, N)[0])


def test_chains_stars_and_parents_that_are_none():
    for parents in ([[i - 1 for i in range(16)]], [[-1] * 16], [[5, 7, -3, 2, 3, 4, 99, 6, 8, 8, -1, 0, 3, 20, 1, 14]]):
        p = ref.Paged([140], [17], 2, 64, b.DOMINO_BF16, 16, seed=5)
        check(p, randq(17, 4, 64, b.DOMINO_BF16, 5), TREE, parents)


@pytest.mark.parametrize("dtype", [b.DOMINO_BF16, b.DOMINO_F32])
def test_rows_that_see_nothing(dtype):
    """kv_len below the new tokens (the first rows lie before every key), tokens past the tree, sequences without keys."""
    p = ref.Paged([5, 64], [9, 20], 2, 64, dtype, 8, seed=6)
    check(p, randq(p.tokens, 4, 64, dtype, 6), CAUSAL)
    check(p, randq(p.tokens, 4, 64, dtype, 6), TREE, ref.random_trees(2, 6, 1)[0])
    p = ref.Paged([0, 3, 0], [4, 1, 2], 2, 64, dtype, 8, seed=7)
    for mask in (CAUSAL, FULL):
        check(p, randq(p.tokens, 4, 64, dtype, 7), mask)


def test_rows_behind_the_last_sequence_and_empty_batches():
    for new in ([3, 0, 2], [0, 0, 0]):
        p = ref.Paged([30, 40, 50], new, 2, 64, b.DOMINO_BF16, 16, seed=8)
        check(p, randq(p.tokens + 5, 4, 64, b.DOMINO_BF16, 8), CAUSAL)


@pytest.mark.parametrize("scale", [1e-3, 0.5, 4.0])
def test_scales(scale):
    """Small scales average, large ones pick one key."""
    p = ref.Paged([900, 300], [40, 7], 2, 128, b.DOMINO_BF16, 32, seed=9)
    check(p, randq(p.tokens, 8, 128, b.DOMINO_BF16, 9), CAUSAL, scale=scale)


@pytest.mark.parametrize("dtype", [b.DOMINO_BF16, b.DOMINO_F16])
def test_growing_scores(dtype):
    """Keys whose scores climb place by place: the running maximum moves with every tile, up and by leaps."""
    p = ref.Paged([1500], [3], 1, 64, dtype, 16, seed=10)
    q = torch.zeros((3, 2, 64), dtype=ref.TORCH[dtype], device=DEV)
    q[:, 0, 0], q[:, 1, 0] = 8.0, -8.0
    at, off = p.slots(0, 1500)
    for climb in (torch.arange(1500, device=DEV) / 4.0, torch.arange(1500, device=DEV) // 128 * 100.0):
        p.k[0, at, off, 0, 0] = climb.to(p.k.dtype)
        check(p, q, CAUSAL)


@pytest.mark.parametrize("dtype", [b.DOMINO_BF16, b.DOMINO_F32])
@pytest.mark.parametrize("mask", [CAUSAL, TREE])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("hq", [4, 32])  # a tile of rows; two of them, and a second group
def test_hidden_new_tokens_do_not_reach_other_rows(dtype, mask, bad, hq):
    """A new token's key and value hold NaN or infinities: rows that see it show them, the others are as without it."""
    p = ref.Paged([200, 300], [20, 20], 2, 64, dtype, 16, seed=11)
    parents = ref.random_trees(2, 19, 3)[0] if mask == TREE else None
    parent = torch.tensor(parents, dtype=torch.int32, device=DEV) if parents else None
    q = randq(p.tokens, hq, 64, dtype, 11)
    clean, _, _ = run(p, q, mask, parent, 19)
    token = 12
    page, off = int(p.table[1, (280 + token) // 16]), (280 + token) % 16
    p.v[0, page, off, 1, 5] = bad
    p.k[0, page, off, 0, 3] = float("nan")
    out, lse, status = run(p, q, mask, parent, 19)
    assert status == 0
    see = ref.visible(mask, 20, 300, parents[1] if parents else None)[:, 280 + token].to(DEV)
    assert torch.equal(out[:20], clean[:20])
    second, was = out[20:], clean[20:]
    assert torch.equal(second[~see], was[~see])
    hit = second[see]
    assert bool(hit[:, :hq // 2].isnan().all()) and bool(lse[20:][see][:, :hq // 2].isnan().all())
    assert bool(hit[:, hq // 2:, 5].isnan().all()) if math.isnan(bad) else bool((hit[:, hq // 2:, 5] == bad).all())
    rest = torch.arange(64, device=DEV) != 5
    assert torch.equal(hit[:, hq // 2:][..., rest], was[see][:, hq // 2:][..., rest])


def test_bad_pages_are_reported():
    p = ref.Paged([100, 300], [2, 2], 2, 64, b.DOMINO_BF16, 16, seed=12)
    q = randq(4, 4, 64, b.DOMINO_BF16, 12)
    clean, _, status = run(p, q, CAUSAL)
    assert status == 0
    for bad in (-1, p.pages, 1 << 30, -(1 << 31)):
        p.table[1, 3] = bad
        out, _, status = run(p, q, CAUSAL)
        assert status == b.DOMINO_ERR_BAD_PAGE and torch.equal(out[:2], clean[:2])


def test_strides_of_queries_and_outputs():
    p = ref.Paged([100, 300], [2, 30], 2, 64, b.DOMINO_BF16, 16, seed=13)
    wide = randq(32, 9, 64, b.DOMINO_BF16, 13)
    q = wide[:, 2:6]
    want = run(p, q.contiguous(), CAUSAL)[0]
    out = torch.full((32, 7, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    n = b.domino_attend_workspace_bytes(32, 4, p.cache)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    args = (p.cache, p.batch, 0.125, CAUSAL, None, 0)
    assert b.domino_attend_paged(q, q.stride(0), 32, 4, *args, out[:, 1:], 7 * 64, None, ws, n, torch.cuda.current_stream()) == 0
    assert torch.equal(out[:, 1:5], want) and bool((out[:, :1] == 7).all()) and bool((out[:, 5:] == 7).all())
    assert b.domino_attend_paged(q, q.stride(0), 32, 4, *args, q, q.stride(0), None, ws, n, torch.cuda.current_stream()) == 0  # in place
    assert torch.equal(q, want)


def test_lengths_out_of_range_are_cut_off():
    p = ref.Paged([48, 64], [4, 4], 2, 64, b.DOMINO_BF16, 16, seed=14)
    q = randq(8, 4, 64, b.DOMINO_BF16, 14)
    want = run(p, q, CAUSAL)[0]
    p.kv_len[1], p.start[2] = 1 << 30, 1 << 30  # the table's four pages, the tensors' eight rows
    assert torch.equal(run(p, q, CAUSAL)[0], want)
    p.kv_len[0] = -5
    out, lse, _ = run(p, q, CAUSAL)
    assert bool((out[:4] == 0).all()) and bool((lse[:4] == -math.inf).all()) and torch.equal(out[4:], want[4:])


def test_the_same_call_gives_the_same_bits_whatever_the_workspace_held():
    p = ref.Paged([3000, 2000, 10], [17, 1, 10], 2, 128, b.DOMINO_BF16, 16, seed=15)
    q = randq(28, 16, 128, b.DOMINO_BF16, 15)
    out, lse, _ = run(p, q, CAUSAL)
    for _ in range(3):
        o, l, _ = run(p, q, CAUSAL)
        assert torch.equal(o, out) and torch.equal(l, lse)


def test_without_lse():
    p = ref.Paged([3000, 10], [17, 1], 2, 128, b.DOMINO_BF16, 16, seed=16)
    q = randq(18, 16, 128, b.DOMINO_BF16, 16)
    assert torch.equal(run(p, q, FULL, lse=False)[0], run(p, q, FULL)[0])


@pytest.mark.parametrize("mask", [CAUSAL, TREE])
def test_many_sequences(mask):
    """More than one launch takes; a bad page of the first launch's sequences shows after the second."""
    n = 1500
    kv = [1 + (i * 37) % 90 for i in range(n)]
    p = ref.Paged(kv, [1 + i % 2 if kv[i] > 1 else i % 2 for i in range(n)], 1, 64, b.DOMINO_BF16, 16, seed=17)
    parents = ref.random_trees(n, 1, 3)[0] if mask == TREE else None
    q = randq(p.tokens, 2, 64, b.DOMINO_BF16, 17)
    check(p, q, mask, parents)
    good = int(p.table[5, 0])
    p.table[5, 0] = -1
    parent = torch.tensor(parents, dtype=torch.int32, device=DEV) if parents else None
    assert run(p, q, mask, parent, 1)[2] == b.DOMINO_ERR_BAD_PAGE
    p.table[5, 0] = good
    check(p, q, mask, parents)


def test_a_long_prompt_in_one_call():
    """9000 tokens from the first place on, 8 heads on one: rows of every group against the 64-bit form."""
    n, hq, D = 9000, 8, 64
    p = ref.Paged([n], [n], 1, D, b.DOMINO_BF16, 64, seed=21)
    q = randq(n, hq, D, b.DOMINO_BF16, 21)
    out, lse, status = run(p, q, CAUSAL)
    assert status == 0
    k, v = p.read(p.k, 0)[:, 0].double(), p.read(p.v, 0)[:, 0].double()
    u = torch.finfo(torch.bfloat16).eps / 2
    for i in sorted({0, 1, 15, 16, 31, 32, 127, 128, 129, 4095, 4096, 8191, 8998, 8999} | set(range(7, n, 613))):
        z = (q[i].double() @ k[:i + 1].T) * D ** -0.5
        l = torch.logsumexp(z, 1)
        w = (z - l[:, None]).exp()
        want, A = w @ v[:i + 1], w @ v[:i + 1].abs()
        e = 2 * (D + 8) * 2.0 ** -24 * (q[i].double().abs() @ k[:i + 1].abs().T).amax(1) * D ** -0.5 + 2.0 ** -20
        assert bool(((out[i].double() - want).abs() <= u * want.abs() + (u + e[:, None]) * A).all()), i
        assert bool(((lse[i].double() - l).abs() <= e / 2 + 2.0 ** -23 * l.abs()).all()), i


def test_offsets_beyond_32_bits():
    """A cache of 2^31 elements and more: pages at its far end."""
    pages, page, hkv, D = 9000, 256, 8, 128
    k = torch.empty((pages, page, hkv, D), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    assert k.numel() > 1 << 31
    g = torch.Generator(device=DEV).manual_seed(18)
    far = [pages - 1, 8300, pages - 2]
    for x in (k, v):
        for f in far:
            x[f] = torch.randn((page, hkv, D), generator=g, device=DEV).bfloat16()
    p = ref.Paged([700], [5], hkv, D, b.DOMINO_BF16, page, seed=18)
    at = p.table[0, :3].long()
    p.k[0, at], p.v[0, at] = k[far], v[far]
    q = randq(5, 16, D, b.DOMINO_BF16, 18)
    want = run(p, q, CAUSAL)[0]
    p.table[0, :3] = torch.tensor(far, dtype=torch.int32)
    s = k.stride()
    p.cache = b.make_cache(k, v, s[0], s[1], s[2], pages, page, hkv, D, b.DOMINO_BF16)
    assert torch.equal(run(p, q, CAUSAL)[0], want)


def test_on_another_stream_and_in_graphs_that_share_a_workspace():
    p = ref.Paged([3000, 200], [17, 17], 2, 128, b.DOMINO_BF16, 16, seed=19)
    qs = [randq(34, 16, 128, b.DOMINO_BF16, 19 + i) for i in range(2)]
    want = [run(p, q, m) for q, m in zip(qs, (CAUSAL, FULL))]
    n = b.domino_attend_workspace_bytes(34, 16, p.cache)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    outs, lses, graphs = [torch.empty_like(q) for q in qs], [torch.empty((34, 16), device=DEV) for _ in qs], []
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for i, m in enumerate((CAUSAL, FULL)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            assert b.domino_attend_paged(qs[i], qs[i].stride(0), 34, 16, p.cache, p.batch, 128 ** -0.5, m, None, 0, outs[i],
                                         outs[i].stride(0), lses[i], ws, n, torch.cuda.current_stream()) == 0
        graphs.append(g)
    for i in (0, 1, 1, 0):
        outs[i].zero_()
        graphs[i].replay()
        assert torch.equal(outs[i], want[i][0]) and torch.equal(lses[i], want[i][1])


def test_short_workspace_is_refused():
    p = ref.Paged([30], [3], 2, 64, b.DOMINO_BF16, 16, seed=20)
    q = randq(3, 4, 64, b.DOMINO_BF16, 20)
    n = b.domino_attend_workspace_bytes(3, 4, p.cache)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    assert b.domino_attend_paged(q, 256, 3, 4, p.cache, p.batch, 1.0, CAUSAL, None, 0, torch.empty_like(q), 256, None, ws, n - 1, None) == \
        b.DOMINO_ERR_INVALID_ARG


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(seed):
    """Any mix of lengths, heads, pages and layouts."""
    g = random.Random(seed)
    dtype, mask = g.choice((b.DOMINO_BF16, b.DOMINO_F16)), g.choice((CAUSAL, FULL, TREE))
    B, hkv, G = g.randint(1, 9), g.randint(1, 4), g.choice((1, 2, 3, 4, 5, 7, 8, 16, 33))
    top = g.choice((1, 5, 40, 70))
    new = [g.randint(0, top) for _ in range(B)]
    kv = [max(0, n + g.choice((-2, 0, 1, 90, 127, 128, 700, 2000)) + g.randint(0, 3)) for n in new]
    N = max(max(new) - g.randint(0, 2), 0)
    p = ref.Paged(kv, new, hkv, 8 * g.randint(1, 16), dtype, 8 * g.choice((1, 2, 3, 5, 8, 16, 17, 32)),
                  g.choice(("pth", "pht", "htp", "thp")), g.choice((0, 8, 24)), seed=seed)
    parents = ref.random_trees(B, N, seed)[0] if mask == TREE else None
    check(p, randq(p.tokens + g.randint(0, 2) + (p.tokens == 0), hkv * G, p.D, dtype, seed), mask, parents)


def test_two_calls_at_once():
    """Two streams, a workspace each: the results of either alone."""
    ps = [ref.Paged([4000, 300], [33, 1], 4, 128, b.DOMINO_BF16, 16, seed=30 + i) for i in range(2)]
    qs = [randq(34, 16, 128, b.DOMINO_BF16, 30 + i) for i in range(2)]
    want = [run(p, q, CAUSAL) for p, q in zip(ps, qs)]
    n = b.domino_attend_workspace_bytes(34, 16, ps[0].cache)
    ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(2)]
    outs, lses = [torch.empty_like(q) for q in qs], [torch.empty((34, 16), device=DEV) for _ in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            assert b.domino_attend_paged(qs[i], qs[i].stride(0), 34, 16, ps[i].cache, ps[i].batch, 128 ** -0.5, CAUSAL, None, 0, outs[i],
                                         outs[i].stride(0), lses[i], ws[i], n, streams[i]) == 0
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], want[i][0]) and torch.equal(lses[i], want[i][1])


def test_a_refused_amount_of_work():
    """Sizes whose line of work does not fit 32 bits are refused before anything is enqueued."""
    p = ref.Paged([30] * 64, [1] * 64, 2, 64, b.DOMINO_BF16, 16, seed=20)  # 64 groups x 2 heads x 3 x 2^24 tiles of the table
    batch = b.make_batch(p.table, 1 << 30, 1 << 30, p.kv_len, p.start, 64)
    q = randq(64, 4, 64, b.DOMINO_BF16, 20)
    n = b.domino_attend_workspace_bytes(64, 4, p.cache)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    assert b.domino_attend_paged(q, 256, 64, 4, p.cache, batch, 1.0, CAUSAL, None, 0, torch.empty_like(q), 256, None, ws, n, None) == \
        b.DOMINO_ERR_UNSUPPORTED
