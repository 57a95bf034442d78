"""Distillation from a teacher's top logits on the GPU (domino_distill_loss / _grad / _loss_grad) against the plain
64-bit form of tests/rows_reference.py.

Bounds.  fp32 throughout: a term exp2((x - m) k2) has an argument of at most 2.5 ulp error (difference, product, k2),
so a relative error of at most (2.5 |t| + 2) 2^-23, t its base-2 logarithm; terms below 2^-30 of the sum do not
matter, so 80 * 2^-23 < 1e-5; a sum of at most 200 sequential terms and 20 tree steps adds 220 * 2^-24 < 1.4e-5 in
the worst case of one sign.  E = 2.5e-5 bounds the relative error of Z and R and the absolute one of their
logarithms, beyond the rounding of values of the size of z (SZ = 2^-22 max |z|).
  loss: |error| <= w (1 + sum q) (E + SZ) + 2^-22 |loss|.
  gradient: |error| <= s [(3 E + SZ) (p_v + rest p_v / p_rest) + 2^-22 q_v], s = w g / T, plus half a step of the
  type: finfo.eps / 2 of the value, and half the smallest subnormal."""
import math

import numpy as np
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import rows_reference as ref
from tests.test_gpu_sample_filtered import DEV, TYPES, logits

pytestmark = pytest.mark.gpu

E = 2.5e-5
F32, BF16, F16 = b.DOMINO_F32, b.DOMINO_BF16, b.DOMINO_F16
RENORM, TAIL = b.DOMINO_DISTILL_RENORM, b.DOMINO_DISTILL_TAIL


def lists(x, kt, mode, T, seed):
    """The teacher: near the student; its best kt ids (fewer where V is smaller: empty places), one row's list with
    an empty place in front, one with an id twice."""
    rows, V = x.shape
    g = torch.Generator().manual_seed(seed)
    t = x.double().cpu() + torch.randn((rows, V), generator=g).double()
    t[t == -math.inf] = -50.0
    t = t / T if mode == TAIL else t
    n = min(kt, V)
    v, i = torch.topk(t, n, dim=1)
    if mode == TAIL:
        v = v - torch.logsumexp(t, 1, keepdim=True)
    ids = torch.full((rows, kt), -1, dtype=torch.int32)
    scores = torch.full((rows, kt), 3.0)
    ids[:, :n], scores[:, :n] = i.int(), v.float()
    if rows > 1 and n > 1:
        ids[1, 0] = -1
    if rows > 2 and n > 2:
        ids[2, 2] = ids[2, 0]
    return ids, scores


def run(part, x, dtype, ids, scores, T, mode, w=None, up=None, pad=0, skew=0, lse=None, inplace=False):
    rows, V = x.shape
    kt = ids.shape[1]
    di, ds = ids.to(DEV), scores.to(DEV)
    dw, du = (None if t is None else t.to(DEV) for t in (w, up))
    loss = torch.full((rows + 2,), 7.0, device=DEV)
    out_lse = torch.full((rows, 2), 7.0, device=DEV) if lse is None else lse
    stride = V + pad
    buf = torch.full((rows * stride + skew + 64,), 5.0, dtype=TYPES[dtype], device=DEV)
    dx = x if inplace else buf[skew:skew + rows * stride].view(rows, stride)[:, :V]
    s = torch.cuda.current_stream()
    if part == "loss":
        rc = b.domino_distill_loss(x, dtype, x.stride(0), di, ds, dw, T, mode, rows, V, kt, loss[1:], out_lse, s)
    elif part == "grad":
        rc = b.domino_distill_grad(x, dtype, x.stride(0), di, ds, dw, du, T, mode, rows, V, kt, out_lse, dx,
                                   dx.stride(0), s)
    else:
        rc = b.domino_distill_loss_grad(x, dtype, x.stride(0), di, ds, dw, du, T, mode, rows, V, kt, loss[1:], out_lse,
                                        dx, dx.stride(0), s)
    assert rc == 0, b.domino_status_string(rc)
    torch.cuda.synchronize()
    if part != "loss" and not inplace:  # what is not an id of a row stays
        whole = buf[skew:skew + rows * stride].view(rows, stride)
        assert (whole[:, V:] == 5.0).all() and (buf[:skew] == 5.0).all() and (buf[skew + rows * stride:] == 5.0).all()
    assert loss[0] == 7.0 and loss[-1] == 7.0
    return loss[1:-1].cpu().double().numpy(), out_lse, dx


def check(x, dtype, ids, scores, T, mode, w, up, loss=None, lse=None, dx=None):
    xs = x.double().cpu().numpy()
    T = float(np.float32(T))
    eps, tiny = torch.finfo(TYPES[dtype]).eps / 2, torch.finfo(TYPES[dtype]).smallest_normal * torch.finfo(TYPES[dtype]).eps / 2
    lse = None if lse is None else lse.cpu().double().numpy()
    g = None if dx is None else dx.double().cpu().numpy()
    for r in range(xs.shape[0]):
        wr, ur = (1.0 if t is None else float(t[r]) for t in (w, up))
        i, s = ids[r].numpy(), scores[r].numpy()
        e, z, rest_lse, eg = ref.distill(xs[r], i, s, T, mode == TAIL, wr, ur)
        zs = xs[r][np.isfinite(xs[r])] / T
        size = 2.0 ** -22 * (np.abs(zs).max() if zs.size else 0.0)
        ok, q, rest = ref.teacher(i, s, xs.shape[1], T, mode == TAIL)
        if loss is not None:
            if np.isinf(e) or e == 0 and wr == 0:
                assert loss[r] == e, (r, loss[r], e)
            else:
                assert abs(loss[r] - e) <= abs(wr) * (1 + q.sum()) * (E + size) + 2.0 ** -22 * abs(e), (r, loss[r], e)
        if lse is not None and wr != 0:
            for got, want in ((lse[r, 0], z), (lse[r, 1], rest_lse)):
                assert got == want if np.isinf(want) else abs(got - want) <= E + size, (r, got, want)
        if g is not None:
            if wr == 0:
                assert (g[r] == 0).all()
                continue
            with np.errstate(invalid="ignore"):
                zz = xs[r] / T
                p = np.exp(zz - z) if z > -np.inf else np.zeros_like(zz)
                pr = rest * np.exp(zz - rest_lse) if rest_lse > -np.inf else np.zeros_like(zz)
            qv = np.zeros_like(p)
            np.add.at(qv, i[ok], q[ok])
            pr[i[ok]] = 0.0
            tol = abs(wr * ur) / T * ((3 * E + size) * (p + pr) + 2.0 ** -22 * qv)
            tol = tol + eps * np.abs(eg) * 1.0001 + tiny
            bad = np.flatnonzero(~(np.abs(g[r] - eg) <= tol))
            assert bad.size == 0, (r, bad[:5], g[r][bad[:5]], eg[bad[:5]], tol[bad[:5]])


SHAPES = [  # rows, V, dtype, kt, T, pad, skew
    (4, 1, F32, 1, 1.0, 0, 0), (3, 2, BF16, 3, 1.0, 1, 1), (4, 37, F16, 5, 0.7, 0, 3), (5, 257, F32, 8, 2.0, 3, 1),
    (4, 999, BF16, 20, 1.0, 0, 0), (3, 4096, F32, 64, 1.5, 0, 0), (3, 5003, F16, 256, 1.0, 5, 5), (6, 33000, BF16, 8, 1.0, 8, 0),
    (3, 33001, F32, 8, 3.0, 0, 0), (2, 151936, BF16, 8, 1.0, 0, 0), (2, 151936, F32, 32, 1.0, 0, 0), (2, 151935, F16, 16, 1.0, 1, 0)]


@pytest.mark.parametrize("mode", [RENORM, TAIL])
@pytest.mark.parametrize("rows,V,dtype,kt,T,pad,skew", SHAPES)
def test_distill_matches_the_plain_form(rows, V, dtype, kt, T, pad, skew, mode):
    x = logits(rows, V, dtype, V + 3, pad=pad, skew=skew)
    ids, scores = lists(x, kt, mode, T, V)
    w = torch.tensor([1.0, 0.5, 0.25, 0.0, 2.0, 1e-3])[:rows]
    up = torch.tensor([3.0, -1.0, 0.5, 1.0, 1.0, 2.0])[:rows]
    loss, lse, _ = run("loss", x, dtype, ids, scores, T, mode, w)
    check(x, dtype, ids, scores, T, mode, w, up, loss, lse)
    _, _, dx = run("grad", x, dtype, ids, scores, T, mode, w, up, pad, skew, lse=lse)
    check(x, dtype, ids, scores, T, mode, w, up, dx=dx)
    loss2, lse2, dx2 = run("both", x, dtype, ids, scores, T, mode, w, up, pad, skew)
    check(x, dtype, ids, scores, T, mode, w, up, loss2, lse2, dx2)
    # gradients into rows of another alignment than the logits'
    for part in ("grad", "both"):
        _, _, dx3 = run(part, x, dtype, ids, scores, T, mode, w, up, pad + 1, skew + 1, lse=lse if part == "grad" else None)
        check(x, dtype, ids, scores, T, mode, w, up, dx=dx3)


@pytest.mark.parametrize("mode", [RENORM, TAIL])
@pytest.mark.parametrize("part", ["grad", "both"])
@pytest.mark.parametrize("dtype,V", [(F32, 20003), (BF16, 40000)])
def test_distill_gradient_in_place(part, mode, dtype, V):
    x = logits(5, V, dtype, 4, pad=1)
    ids, scores = lists(x, 16, mode, 1.0, 4)
    _, lse, want = run("both", x, dtype, ids, scores, 1.0, mode)
    if part == "grad":
        _, _, want = run("grad", x, dtype, ids, scores, 1.0, mode, lse=lse)
    y = logits(5, V, dtype, 4, pad=1)  # the same rows at the same alignment
    _, _, got = run(part, y, dtype, ids, scores, 1.0, mode, lse=lse if part == "grad" else None, inplace=True)
    assert got.data_ptr() == y.data_ptr() and torch.equal(got, want)


@pytest.mark.parametrize("mode", [RENORM, TAIL])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_distill_masked_logits_and_empty_lists(dtype, mode):
    """-inf and the type's lowest value in masked places, rows without a logit, listed ids that are masked, lists
    without an id, lists that hold every id, far-off listed logits, rows of weight 0 that hold NaN."""
    V, kt = 300, 8
    x = logits(11, V, dtype, 21)
    ids, scores = lists(x, kt, mode, 1.0, 21)
    x[0, 100:] = -math.inf
    ids[0] = torch.arange(kt).int() * 10
    x[1, 50:] = torch.finfo(TYPES[dtype]).min
    ids[1] = torch.arange(kt).int()
    x[2] = -math.inf
    ids[3] = -1
    x[4, ids[4].long()] = -math.inf
    x[5] = math.nan
    ids[6, 3:] = V + 5  # outside: empty
    scores[6, 1] = -math.inf
    x[7, ids[7].long()] += 30.0  # the rest is far below
    x[8, ids[8, 0].long()] = 200.0 if dtype == F16 else 3000.0
    x[9], ids[9] = -math.inf, -1
    x[10, kt:] = -math.inf  # nothing but listed ids
    ids[10] = torch.arange(kt).int()
    w = torch.ones(11)
    w[5] = 0.0
    up = torch.ones(11)
    loss, lse, _ = run("loss", x, dtype, ids, scores, 1.0, mode, w)
    check(x, dtype, ids, scores, 1.0, mode, w, up, loss, lse)
    _, _, dx = run("grad", x, dtype, ids, scores, 1.0, mode, w, up, lse=lse)
    check(x, dtype, ids, scores, 1.0, mode, w, up, dx=dx)
    loss, lse, dx = run("both", x, dtype, ids, scores, 1.0, mode, w, up)
    check(x, dtype, ids, scores, 1.0, mode, w, up, loss, lse, dx)


def test_distill_nan_shows():
    """A NaN logit of a weighted row makes its loss NaN instead of being passed over."""
    x = logits(3, 1000, F32, 22)
    ids, scores = lists(x, 4, TAIL, 1.0, 22)
    x[0, 700] = math.nan
    x[1, ids[1, 1].long()] = math.nan
    loss, lse, dx = run("both", x, F32, ids, scores, 1.0, TAIL)
    assert np.isnan(loss[:2]).all() and np.isfinite(loss[2])
    assert torch.isnan(dx[:2]).any(1).all() and torch.isfinite(dx[2]).all()


@pytest.mark.parametrize("mode", [RENORM, TAIL])
def test_distill_nan_scores_show(mode):
    """A NaN among the teacher's scores makes the row's loss NaN, and its gradient by every entry point."""
    x = logits(3, 1000, F32, 28)
    ids, scores = lists(x, 4, mode, 1.0, 28)
    scores[0, 1] = math.nan
    scores[1] = math.nan
    loss, lse, dx = run("both", x, F32, ids, scores, 1.0, mode)
    _, _, dx2 = run("grad", x, F32, ids, scores, 1.0, mode, lse=lse)
    assert np.isnan(loss[:2]).all() and np.isfinite(loss[2])
    for d in (dx, dx2):
        assert torch.isnan(d[:2]).any(1).all() and torch.isfinite(d[2]).all()


@pytest.mark.parametrize("mode", [RENORM, TAIL])
def test_distill_gradient_is_the_loss_difference(mode):
    """Central differences of the loss that the GPU returns: step h = 2^-5, error of the quotient h^2 / 6 times the
    third derivative (at most 1 for a softmax at T >= 1, both terms: 2) plus two losses' rounding (E each) over 2 h."""
    V, T, h = 60, 1.3, 2.0 ** -5
    x = logits(1, V, F32, 23, std=1.0)
    ids, scores = lists(x, 6, mode, T, 23)
    _, _, dx = run("both", x, F32, ids, scores, T, mode)
    y = x.expand(2 * V, V).clone()
    y[:V] += h * torch.eye(V, device=DEV)
    y[V:] -= h * torch.eye(V, device=DEV)
    loss, _, _ = run("loss", y, F32, ids.expand(2 * V, -1).contiguous(), scores.expand(2 * V, -1).contiguous(), T, mode)
    quotient = (loss[:V] - loss[V:]) / (2 * h)
    assert np.all(np.abs(quotient - dx[0].double().cpu().numpy()) <= 2 * h * h / 6 + 2 * E / (2 * h))


def test_distill_defaults_and_largest_vocabulary():
    """No weights, no upstream gradient, no lse output; the largest V."""
    V = 1 << 19
    for dtype in (F32, BF16):
        x = logits(2, V, dtype, 24)
        ids, scores = lists(x, 8, TAIL, 1.0, 24)
        loss, lse, dx = run("both", x, dtype, ids, scores, 1.0, TAIL)
        check(x, dtype, ids, scores, 1.0, TAIL, None, None, loss, lse, dx)
        only = torch.empty(2, device=DEV)
        assert b.domino_distill_loss(x, dtype, V, ids.to(DEV), scores.to(DEV), None, 1.0, TAIL, 2, V, 8, only, None,
                                     torch.cuda.current_stream()) == 0
        check(x, dtype, ids, scores, 1.0, TAIL, None, None, only.cpu().double().numpy())


def test_distill_beyond_32_bit_offsets():
    V, stride = 3000, (1 << 31) + 8
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (3, V), (stride, 1))
    x.copy_(logits(3, V, BF16, 25))
    ids, scores = lists(x, 8, TAIL, 1.0, 25)
    loss, lse, dx = run("both", x, BF16, ids, scores, 1.0, TAIL)
    check(x, BF16, ids, scores, 1.0, TAIL, None, None, loss, lse, dx)
    run("grad", x, BF16, ids, scores, 1.0, TAIL, lse=lse, inplace=True)  # and written there
    assert torch.allclose(x.float(), dx.float(), atol=1e-5, rtol=2.0 ** -7)


def test_distill_in_a_graph_and_repeats():
    """A captured loss and gradient, replayed on new logits; the same bits from the same inputs."""
    V, rows = 30011, 40
    x = logits(rows, V, BF16, 26)
    ids, scores = lists(x, 8, TAIL, 1.0, 26)
    di, ds = ids.to(DEV), scores.to(DEV)
    loss, lse, dx = torch.empty(rows, device=DEV), torch.empty((rows, 2), device=DEV), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert b.domino_distill_loss_grad(x, BF16, V, di, ds, None, None, 1.0, TAIL, rows, V, 8, loss, lse, dx, V,
                                          torch.cuda.current_stream()) == 0
    x.copy_(logits(rows, V, BF16, 27))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    l2, lse2, dx2 = run("both", x, BF16, ids, scores, 1.0, TAIL)
    assert (loss.cpu().double().numpy() == l2).all() and torch.equal(lse, lse2) and torch.equal(dx, dx2)
    check(x[:3], BF16, ids[:3], scores[:3], 1.0, TAIL, None, None, l2, lse2, dx2[:3])
