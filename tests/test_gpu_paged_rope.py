"""Rotary positions, alone and with the write into a paged cache, against their fp64 forms."""
import math

import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
LAYOUTS = [b.DOMINO_ROPE_HALF, b.DOMINO_ROPE_PAIRS]
TYPES = [b.DOMINO_F32, b.DOMINO_BF16, b.DOMINO_F16]


def speeds(rot, factor=1.0):
    half = rot // 2
    return torch.tensor([1e6 ** (-i / half) / factor for i in range(half)], dtype=torch.float32, device=DEV)


def randn(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(ref.TORCH[dtype])


def rope(x, dtype, pos, freq, amplitude, layout, gradient, rot, y):
    t, h, D = x.shape
    return b.domino_rope(x, dtype, x.stride(0), x.stride(1), pos, freq, amplitude, layout, gradient, t, h, D, rot, y, y.stride(0),
                         y.stride(1), torch.cuda.current_stream())


def close(y, want, tol):
    err = (y.double() - want).abs()
    assert bool((err <= tol).all()), float((err - tol).max())


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,heads,D,rot", [(1, 1, 2, 2), (1, 32, 128, 128), (17, 5, 80, 40), (33, 3, 80, 80), (130, 2, 96, 48),
                                                (7, 4, 64, 0), (5, 3, 7, 6), (3, 1, 255, 254), (64, 2, 256, 128), (700, 9, 128, 64)])
def test_rope(layout, dtype, tokens, heads, D, rot):
    x = randn((tokens, heads, D), dtype, tokens + D)
    pos = torch.randint(0, 40000, (tokens,), device=DEV, dtype=torch.int32, generator=torch.Generator(device=DEV).manual_seed(1))
    freq = speeds(rot) if rot else None
    for back in (False, True):
        y = torch.full_like(x, float("nan"))
        assert rope(x, dtype, pos, freq, 1.25, layout, int(back), rot, y) == 0
        want, tol = ref.rotate(x, pos, freq if rot else torch.zeros(0, device=DEV), rot, layout, 1.25, back)
        close(y, want, tol)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_far_negative_and_strange_positions(layout):
    pos = torch.tensor([0, 1, -1, 1 << 20, -(1 << 20), (1 << 31) - 1, -(1 << 31), 123456789, -987654321], dtype=torch.int32, device=DEV)
    freq = torch.tensor([1.0, 0.5, 1e-6, 1e-30, 0.0, -0.7, math.pi, 1024.0, 1000.123, 3.1e-39, 6.2831855, 1.0 / 3, 0.9999999, 2e-9,
                         77.7, -1024.0], device=DEV)
    x = randn((pos.numel(), 3, 32), b.DOMINO_F32, 3)
    y = torch.empty_like(x)
    assert rope(x, b.DOMINO_F32, pos, freq, 1.0, layout, 0, 32, y) == 0
    # the fp64 product of position and speed, up to 2^41 radians, is itself off by 2^-53 of that: 2^-12
    z = pos.double()[:, None] * freq.double()
    want, tol = ref.rotate(x, pos, freq, 32, layout, 1.0)
    # the device's speed in turns is cut at 2^-64 (2^-62 of a speed above a turn a position): |position| 2^-62 max(1, speed)
    slack = z.abs() * 2.0 ** -52 + pos.double().abs()[:, None] * 2.0 ** -59 * freq.double().abs().clamp(min=1.0)
    i = torch.arange(16, device=DEV)
    at = torch.cat((i, i)) if layout == b.DOMINO_ROPE_HALF else i.repeat_interleave(2)
    close(y, want, tol + (slack[:, at])[:, None] * x.double().abs().amax() * 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,head_pad,shift", [(8, 0, 0), (4, 4, 4), (3, 1, 1), (16, 8, 8)])
def test_strides_and_alignment(dtype, pad, head_pad, shift):
    tokens, heads, D, rot = 29, 3, 64, 32
    store = randn((tokens * (heads * (D + head_pad) + pad) + shift,), dtype, 9)
    x = torch.as_strided(store, (tokens, heads, D), (heads * (D + head_pad) + pad, D + head_pad, 1), shift)
    out = torch.full((heads, tokens, D + pad), 7.0, dtype=x.dtype, device=DEV)
    y = out.permute(1, 0, 2)[..., :D]  # heads outside
    pos = torch.arange(tokens, dtype=torch.int32, device=DEV) * 100
    assert rope(x, dtype, pos, speeds(rot), 1.0, b.DOMINO_ROPE_HALF, 0, rot, y) == 0
    want, tol = ref.rotate(x, pos, speeds(rot), rot, b.DOMINO_ROPE_HALF, 1.0)
    close(y, want, tol)
    assert bool((out[..., D:] == 7.0).all())


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("D,rot", [(128, 128), (80, 40), (65, 32)])
def test_in_place(layout, D, rot):
    x = randn((200, 4, D), b.DOMINO_BF16, 4)
    pos = torch.arange(200, dtype=torch.int32, device=DEV)
    y = torch.empty_like(x)
    assert rope(x, b.DOMINO_BF16, pos, speeds(rot), 1.0, layout, 0, rot, y) == 0
    assert rope(x, b.DOMINO_BF16, pos, speeds(rot), 1.0, layout, 0, rot, x) == 0
    assert torch.equal(x, y)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_the_gradient_is_the_transpose_and_agrees_with_differences(layout):
    tokens, heads, D, rot = 6, 2, 32, 24
    x, w = randn((tokens, heads, D), b.DOMINO_F32, 5), randn((tokens, heads, D), b.DOMINO_F32, 6)
    pos = torch.tensor([0, 3, 1 << 20, 17, 999, 65535], dtype=torch.int32, device=DEV)
    g, y0, y1 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    assert rope(w, b.DOMINO_F32, pos, speeds(rot), 1.5, layout, 1, rot, g) == 0
    step = randn((tokens, heads, D), b.DOMINO_F32, 7)
    assert rope(x + step, b.DOMINO_F32, pos, speeds(rot), 1.5, layout, 0, rot, y1) == 0
    assert rope(x - step, b.DOMINO_F32, pos, speeds(rot), 1.5, layout, 0, rot, y0) == 0
    # the map is linear: the difference of sum(w y) over two steps is that of its gradient along the step, up to the
    # roundings of y (4 2^-23 1.5 of two elements each, as in ref.rotate) and of x +- step (2^-24)
    slope = float((w.double() * (y1.double() - y0.double())).sum() / 2)
    size = float((w.double().abs().amax() * (x.abs() + step.abs()).double().sum())) * 2
    assert abs(slope - float((g.double() * step.double()).sum())) <= size * 1.5 * 5 * 2.0 ** -23


def _append(p, dtype, hq, layout, rot, depth=None, N=0, positions=None, pad=0, queries=True, in_place=False, seed=3):
    """Runs the call on one projection's output; checks q, the cache, and that nothing else changed."""
    wide = (hq + 2 * p.hkv) * p.D
    qkv = randn((p.tokens, wide + pad), dtype, seed)
    q, k, v, _ = qkv.split((hq * p.D, p.hkv * p.D, p.hkv * p.D, pad), 1)
    q, k, v = (t.unflatten(1, (-1, p.D)) for t in (q, k, v))
    want_q_in = q.clone()
    freq = speeds(rot, 4.0)
    q_out = q if in_place else torch.full((p.tokens, hq, p.D), float("nan"), dtype=qkv.dtype, device=DEV)
    k_was, v_was = p.k_store.clone(), p.v_store.clone()
    rc = b.domino_rope_append(q if queries else None, qkv.stride(0), k, qkv.stride(0), v, qkv.stride(0), positions, depth, N, freq, 1.125,
                              layout, rot, hq if queries else 0, p.tokens, q_out if queries else None, q_out.stride(0), p.cache,
                              p.batch, torch.cuda.current_stream())
    assert rc == 0
    seq, place, pos = [], [], []
    for i in range(p.B):
        for t in range(p.new[i]):
            at = p.kv[i] - p.new[i] + t
            seq.append(i)
            place.append(at)
            pos.append(p.kv[i] - p.new[i] + int(depth[i, t - 1]) if depth is not None and 1 <= t <= N else at)
    pos = torch.tensor(pos, device=DEV) if positions is None else positions[:len(pos)]
    n = len(seq)  # rows behind the last sequence stay
    want, tol = ref.rotate(want_q_in[:n], pos, freq, rot, layout, 1.125)
    if queries:
        close(q_out[:n], want, tol)
    want, tol = ref.rotate(k[:n], pos, freq, rot, layout, 1.125)
    seen = torch.zeros(p.k.shape[1:3], dtype=torch.bool, device=DEV)
    for r in range(n):
        if place[r] < 0:
            continue
        page = int(p.table[seq[r], place[r] // p.page])
        if not 0 <= page < p.pages:
            continue
        at = place[r] % p.page
        close(p.k[0, page, at], want[r], tol[r])
        assert torch.equal(p.v[0, page, at], v[r])
        seen[page, at] = True
    same = lambda now, was: (now == was) | (now.isnan() & was.isnan())
    perm_k, perm_v = torch.as_strided(k_was, p.k.shape, p.k.stride()), torch.as_strided(v_was, p.v.shape, p.v.stride())
    assert bool(same(p.k[0], perm_k[0])[~seen].all()) and bool(same(p.v[0], perm_v[0])[~seen].all())
    return q_out, n


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("order,page,D,rot,pad,kpad", [("pth", 16, 128, 128, 0, 0), ("pht", 48, 128, 64, 64, 0), ("htp", 1, 80, 40, 4, 4),
                                                       ("pth", 7, 65, 32, 3, 1), ("pht", 256, 96, 96, 8, 8)])
def test_append(dtype, layout, order, page, D, rot, pad, kpad):
    p = ref.Paged([300, 5, 33, 64], [37, 5, 0, 1], 2, D, dtype, page, order, kpad, seed=8)
    _append(p, dtype, 6, layout, rot, pad=pad)


def test_append_a_single_token_and_a_long_chunk():
    for kv, new in (([1], [1]), ([2048, 100], [1500, 1]), ([5000] * 40, [1] * 40)):
        p = ref.Paged(kv, new, 8, 128, b.DOMINO_BF16, 32, seed=9)
        _append(p, b.DOMINO_BF16, 32, b.DOMINO_ROPE_HALF, 128)


def test_append_trees_by_depth():
    N = 16
    p = ref.Paged([50, 17, 400], [17, 17, 12], 4, 64, b.DOMINO_F16, 16, seed=10)
    _, depth = ref.random_trees(3, N, 5)
    _append(p, b.DOMINO_F16, 8, b.DOMINO_ROPE_HALF, 64, torch.tensor(depth, dtype=torch.int32, device=DEV), N)


def test_append_given_positions_keys_alone_and_in_place():
    p = ref.Paged([50, 9], [10, 9], 4, 64, b.DOMINO_BF16, 16, seed=11)
    pos = torch.randint(-1000, 1 << 20, (19,), device=DEV, dtype=torch.int32)
    _append(p, b.DOMINO_BF16, 8, b.DOMINO_ROPE_PAIRS, 64, positions=pos)
    _append(p, b.DOMINO_BF16, 8, b.DOMINO_ROPE_PAIRS, 64, queries=False, seed=12)
    _append(p, b.DOMINO_BF16, 8, b.DOMINO_ROPE_PAIRS, 64, in_place=True, seed=13)


def test_append_leaves_out_places_without_a_page_and_rows_behind_the_last_sequence():
    p = ref.Paged([50, 9, 3], [10, 9, 3], 4, 64, b.DOMINO_BF16, 4, seed=14)
    p.table[0, 11] = -1          # places 44 .. 47
    p.table[1, 1] = p.pages + 3  # places 4 .. 7
    p.start[3] = 20              # the last sequence has one token, its last place; two rows are nobody's
    p.new[2], p.start_host[3] = 1, 20
    q_out, n = _append(p, b.DOMINO_BF16, 8, b.DOMINO_ROPE_HALF, 64, seed=15)
    assert n == 20 and bool(q_out[20:].isnan().all())


def test_lengths_out_of_range_touch_nothing_outside():
    """kv_len beyond the table and starts beyond the rows are cut off; places before the first are not written."""
    p = ref.Paged([8, 8], [4, 4], 2, 64, b.DOMINO_BF16, 4, seed=16)
    p.kv_len[0], p.kv_len[1] = 1 << 30, 2
    p.start[2] = 1000
    p.kv, p.new = [8, 2], [4, 4]
    _append(p, b.DOMINO_BF16, 4, b.DOMINO_ROPE_HALF, 64, seed=17)


def test_a_captured_call_follows_its_inputs():
    p = ref.Paged([40, 90], [3, 20], 2, 64, b.DOMINO_BF16, 16, seed=18)
    x = randn((23, 4, 64), b.DOMINO_BF16, 1)
    kv = randn((23, 2, 64), b.DOMINO_BF16, 2)
    y, freq = torch.empty_like(x), speeds(64)

    def call():
        assert b.domino_rope_append(x, x.stride(0), kv, kv.stride(0), kv, kv.stride(0), None, None, 0, freq, 1.0, b.DOMINO_ROPE_HALF, 64,
                                    4, 23, y, y.stride(0), p.cache, p.batch, torch.cuda.current_stream()) == 0

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
    p.kv_len -= 2
    x.copy_(randn((23, 4, 64), b.DOMINO_BF16, 3))
    graph.replay()
    pos = torch.tensor([35 + i for i in range(3)] + [68 + i for i in range(20)], device=DEV)
    want, tol = ref.rotate(x, pos, freq, 64, b.DOMINO_ROPE_HALF, 1.0)
    close(y, want, tol)
