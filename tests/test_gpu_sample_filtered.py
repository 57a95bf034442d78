"""Draws after temperature, top-k, top-p and min-p on the GPU (domino_sample_filtered) against the plain
64-bit form of tests/rows_reference.py.

The token has to be the plain form's wherever the plain form's nearest border (of top-p, of u) is more than
BORDER of the mass away.  The kernel's weights are off by at most 2^-44 of the greatest (their last places) plus
2^-37 of their value where they are above 2^-11 of it, and 2^-19 of their value (fp32: the argument's rounding, up
to 45 * 2^-24, and the exponential's) below; under top-p what cannot stay is summed in fp32 by some thousand threads
of a few hundred terms each, 2^-20 of that mass per thread at most.  The errors of different ids and threads are
independent and of either sign: n of them that carry a share s of the mass move a border by about s 2^-19 / sqrt(n).
With s below 1/2 and n in the thousands that stays under 3e-8 of the mass; the exact weights contribute 2^-37 and
V 2^-44 < 3e-8 in the worst case of one sign.  BORDER = 1e-7; rows that close to a border (one in some hundred
thousand uniforms) may give either neighbour, and none of the seeds here may put more than one such row into a case.

logp: fp32.  z carries two roundings (subtraction, division) and log(mass) one of the sum, the logarithm's
(1 ulp) and the subtraction's: |error| <= 2^-23 |z| + 2^-23 log(mass) + 2^-24 |logp| + 2^-24 < 2^-21 (1 + |logp| +
log V)."""
import math

import numpy as np
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import rows_reference as ref

pytestmark = pytest.mark.gpu

BORDER = 1e-7
DEV = "cuda:0"
TYPES = {b.DOMINO_F32: torch.float32, b.DOMINO_BF16: torch.bfloat16, b.DOMINO_F16: torch.float16}
F32, BF16, F16 = b.DOMINO_F32, b.DOMINO_BF16, b.DOMINO_F16


def dev(values, dtype):
    return None if values is None else torch.tensor(values, dtype=dtype, device=DEV)


def logits(rows, V, dtype, seed, std=4.0, pad=0, skew=0):
    """[rows, V] in memory of row stride V + pad whose first element lies `skew` elements into a buffer; the
    padding is +inf (reading it would show)."""
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((rows * (V + pad) + skew + 64,), math.inf, dtype=TYPES[dtype])
    x = buf[skew:skew + rows * (V + pad)].view(rows, V + pad)
    x[:, :V] = (torch.randn((rows, V), generator=g) * std).to(TYPES[dtype])
    d = buf.to(DEV)
    return d[skew:skew + rows * (V + pad)].view(rows, V + pad)[:, :V]


def uniforms(rows, seed):
    return torch.rand(rows, generator=torch.Generator().manual_seed(1000 + seed))


def run(x, dtype, u, T=None, k=None, p=None, m=None, logp=True, stream=None):
    rows, V = x.shape
    out = torch.full((rows + 2,), -7, dtype=torch.int32, device=DEV)
    lp = torch.full((rows + 2,), 7.0, device=DEV)
    keep = [dev(T, torch.float32), dev(k, torch.int32), dev(p, torch.float32), dev(m, torch.float32), u.to(DEV)]
    rc = b.domino_sample_filtered(x, dtype, x.stride(0), *keep, rows, V, out[1:], lp[1:] if logp else None,
                                  stream or torch.cuda.current_stream())
    assert rc == 0, b.domino_status_string(rc)
    torch.cuda.synchronize()
    out, lp = out.cpu().numpy(), lp.cpu().numpy()
    assert out[0] == -7 and out[-1] == -7 and lp[0] == 7.0 and lp[-1] == 7.0  # the neighbours, as they were
    return out[1:-1], lp[1:-1]


def check(x, u, got, lp, T=None, k=None, p=None, m=None):
    xs = x.double().cpu().numpy()
    close = 0
    for r in range(xs.shape[0]):
        a = dict(T=1.0 if T is None else float(np.float32(T[r])), k=0 if k is None else k[r],
                 p=1.0 if p is None else float(np.float32(p[r])), m=0.0 if m is None else float(np.float32(m[r])))
        e, elp, margin = ref.draw(xs[r], float(u[r]), **a)
        if margin < BORDER and got[r] != e:
            close += 1
            continue
        assert got[r] == e, (r, a, float(u[r]), int(got[r]), e, margin)
        if lp is not None:
            if np.isinf(elp):
                assert lp[r] == elp
            else:
                assert abs(lp[r] - elp) <= 2.0 ** -21 * (1 + abs(elp) + math.log(xs.shape[1])), (r, lp[r], elp)
    assert close <= 1


def run_and_check(x, dtype, u, **a):
    """The rows by themselves (few: one kernel for latency), and four times over (many: the other)."""
    got, lp = run(x, dtype, u, **a)
    check(x, u, got, lp, **a)
    rows, V = x.shape
    stride, skew = x.stride(0), x.storage_offset()
    buf = torch.empty(4 * rows * stride + skew, dtype=x.dtype, device=DEV)
    y = torch.as_strided(buf, (4 * rows, V), (stride, 1), skew)
    y.copy_(x.repeat(4, 1))
    got, lp = run(y, dtype, u.repeat(4), **{k: v * 4 for k, v in a.items()})
    for i in (0, 3):
        check(x, u, got[i * rows:(i + 1) * rows], lp[i * rows:(i + 1) * rows], **a)
    return got[:rows], lp[:rows]


RULES = {
    "none": {},
    "temp": dict(T=[0.7, 1.0, 1.6, 0.3, 3.0, 0.05]),
    "topk": dict(T=[0.7, 1.0, 1.6, 0.3, 3.0, 1.0], k=[1, 2, 5, 50, 200, 700]),
    "topp": dict(T=[0.7, 1.0, 1.6, 0.3, 3.0, 1.0], p=[0.9, 0.5, 0.99, 0.05, 0.95, 0.999]),
    "minp": dict(T=[0.7, 1.0, 1.6, 0.3, 3.0, 1.0], m=[0.1, 0.5, 0.01, 0.05, 0.3, 1e-6]),
    "topk-topp": dict(T=[0.7, 1.0, 1.6, 0.3, 3.0, 1.0], k=[50, 3, 1000, 40, 20, 100], p=[0.9, 0.5, 0.99, 0.8, 0.3, 0.95]),
    "topp-minp": dict(p=[0.9, 0.5, 0.99, 0.8, 0.3, 0.95], m=[0.1, 0.001, 0.01, 0.5, 0.3, 1e-5]),
    "all": dict(T=[0.7, 1.0, 1.6, 0.3, 3.0, 0.0], k=[50, 0, 1000, 40, -1, 100], p=[0.9, 1.0, 0.99, 0.8, 0.3, 0.95],
                m=[0.0, 0.1, 0.01, 0.05, 0.02, 0.1]),
}


@pytest.mark.parametrize("rule", sorted(RULES))
@pytest.mark.parametrize("dtype,V,pad,skew", [
    (F32, 1, 0, 0), (F16, 1, 3, 1), (F32, 2, 0, 0), (BF16, 5, 1, 0), (F32, 8, 0, 0), (F16, 37, 0, 3), (F32, 257, 0, 1),
    (BF16, 999, 1, 0), (F32, 4096, 0, 0), (BF16, 4096, 0, 0), (F32, 5003, 5, 2), (F16, 5003, 5, 5), (BF16, 33000, 8, 0),
    (F32, 33001, 0, 0)])
def test_draw_matches_the_plain_form(rule, dtype, V, pad, skew):
    x = logits(6, V, dtype, V + 11, pad=pad, skew=skew)
    u = uniforms(6, V)
    run_and_check(x, dtype, u, **RULES[rule])


@pytest.mark.parametrize("rule", sorted(RULES))
@pytest.mark.parametrize("dtype,V", [(F32, 151936), (BF16, 151936), (F16, 151935)])
def test_draw_full_vocabulary(rule, dtype, V):
    x = logits(6, V, dtype, 77, std=5.1)
    u = uniforms(6, 77)
    run_and_check(x, dtype, u, **RULES[rule])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("std,rule", [(0.0, "topk"), (0.0, "topp"), (0.0, "minp"), (0.02, "topp"), (0.5, "topk-topp"),
                                      (0.5, "topp"), (1.0, "minp"), (0.5, "none"), (40.0, "all"), (1.0, "topp-minp")])
def test_draw_flat_and_sharp_rows(dtype, std, rule):
    """Rows of equal logits, rows so flat that most of the vocabulary stays, and rows with one survivor."""
    x = logits(6, 40003, dtype, 5, std=std)
    u = uniforms(6, 5)
    run_and_check(x, dtype, u, **RULES[rule])


@pytest.mark.parametrize("dtype,V", [(F32, 1 << 19), (BF16, (1 << 19) - 3)])
def test_draw_largest_vocabulary(dtype, V):
    x = logits(6, V, dtype, 6, std=3.0)
    u = uniforms(6, 6)
    for rule in ("none", "all"):
        run_and_check(x, dtype, u, **RULES[rule])


@pytest.mark.parametrize("rule", ["topk", "topp", "all", "none"])
def test_draw_ties(rule):
    """Logits on a coarse grid: every cut falls among equal values, and the lower ids stay."""
    x = (logits(6, 20011, F32, 8, std=1.5) * 2).round() / 2  # -0 among them
    u = uniforms(6, 8)
    for t, y in ((F32, x), (BF16, x.bfloat16())):
        run_and_check(y.contiguous(), t, u, **RULES[rule])


@pytest.mark.parametrize("order", ["rising", "falling"])
@pytest.mark.parametrize("rule", ["topk", "topp", "all"])
def test_draw_sorted_rows(order, rule):
    """All candidates side by side: at one end of the vocabulary."""
    x = logits(6, 30000, F32, 9).sort(dim=1, descending=order == "falling").values.contiguous()
    u = uniforms(6, 9)
    run_and_check(x, F32, u, **RULES[rule])


@pytest.mark.parametrize("rule", ["topk", "topp", "minp", "all"])
@pytest.mark.parametrize("dtype,V", [(F32, 151936), (BF16, 151935)])
def test_draw_rows_that_a_sample_misjudges(rule, dtype, V):
    """Long rows whose sample says little: sorted ones (all candidates in a few warps' ids), one token far above the
    rest, a few finite logits among -inf and NaN, a run of high logits, two levels only, a plateau under a peak."""
    x = logits(6, V, dtype, 31, std=3.0)
    x[0] = x[0].sort().values
    x[1] = x[1].sort(descending=True).values
    x[2, 77777] = 60.0
    x[3] = -math.inf
    x[3, [5, 77777, V - 1]] = torch.tensor([1.0, 2.0, 1.5], device=DEV).to(TYPES[dtype])
    x[3, 100:200] = math.nan
    x[4] = x[4].clamp(max=4.0)
    x[4, 40000:46000] = 9.0  # more equal candidates than any list holds
    x[5] = 0.0
    x[5, ::3] = 1.0
    u = uniforms(6, 31)
    run_and_check(x, dtype, u, **RULES[rule])


def test_draw_masked_and_infinite_logits():
    """-inf, NaN and the type's lowest value in masked places, rows without any logit, +inf."""
    V = 3001
    for dtype in (F32, BF16, F16):
        x = logits(10, V, dtype, 12)
        x[0, :1500] = -math.inf
        x[1, ::2] = math.nan
        x[2, 7:] = -math.inf
        x[3] = -math.inf
        x[4] = math.nan
        x[5] = torch.finfo(TYPES[dtype]).min
        x[6, 100:] = torch.finfo(TYPES[dtype]).min
        x[7, [5, 1000, 2999]] = math.inf
        x[8, :] = -math.inf
        x[8, 2500] = -3.0
        x[9, 1] = math.inf
        x[9, 2] = math.nan
        u = uniforms(10, 12)
        for a in ({}, dict(k=[40] * 10), dict(p=[0.9] * 10), dict(m=[0.05] * 10), dict(T=[0.0] * 10),
                  dict(T=[0.5] * 10, k=[2000] * 10, p=[0.8] * 10, m=[0.01] * 10)):
            got, lp = run_and_check(x, dtype, u, **a)
            assert got[3] == 0 and got[4] == 0 and lp[3] == -math.inf


def test_draw_extreme_settings():
    """Settings outside their range turn a filter off, or leave the first id."""
    V, n = 2003, 12
    x = logits(n, V, F32, 13)
    u = uniforms(n, 13)
    inf, nan = math.inf, math.nan
    a = dict(T=[0.0, -1.0, nan, 1e-40, 1e-30, 1e30, inf, 1.0, 1.0, 1.0, 1.0, 1.0],
             k=[0, 0, 0, 0, 0, 0, 0, -5, V, V + 9, 2 ** 31 - 1, 1],
             p=[1.0, 0.5, 0.5, 0.5, 0.5, 1.0, 1.0, 0.0, -1.0, nan, 1.5, 1e-20],
             m=[0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, nan, -2.0, 5.0])
    got, lp = run(x, F32, u, **a)
    top = x.argmax(1).cpu().numpy()
    for r in (0, 1, 2, 3, 4, 7, 8, 11):
        assert got[r] == top[r] and lp[r] == 0.0, r
    for r in (5, 6):  # infinitely hot: every id as likely as any other
        assert got[r] == int(float(u[r]) * V) and abs(lp[r] + math.log(V)) < 1e-5
    full, _ = run(x, F32, u)
    assert (got[9:11] == full[9:11]).all()
    one, _ = run(x, F32, u, p=[1.0] * n, m=[1.0] * n)
    assert (one == top).all()


@pytest.mark.parametrize("dtype,V", [(F32, 151935), (BF16, 151935), (F32, 901), (F16, 40003)])
def test_draw_infinitely_hot_rows_with_masked_ids(dtype, V):
    """T = inf makes the ids that are not masked equally likely; -inf, whose product with 1 / T has no value, stays out
    of the draw and out of the mass that top-p goes by."""
    x = logits(6, V, dtype, 32)
    x[0, ::2] = -math.inf
    x[1, V // 3:] = -math.inf
    x[2, : V // 3] = -math.inf
    x[3, 7] = -math.inf
    x[4, ::3] = math.nan
    u = uniforms(6, 32)
    T = [math.inf] * 6
    for a in (dict(), dict(p=[0.9, 0.3, 0.99, 0.5, 0.05, 0.7]), dict(k=[50] * 6, p=[0.71] * 6), dict(k=[50] * 6),
              dict(m=[0.5] * 6), dict(p=[0.63] * 6, m=[0.5] * 6)):
        run_and_check(x, dtype, u, T=T, **a)


def test_draw_interval_ends():
    """u on the borders of four equal ids, at the ends of [0, 1), and outside."""
    x = torch.zeros((9, 4), device=DEV)
    u = torch.tensor([0.0, 0.25, 0.5, 0.75, ref.BELOW_ONE, -0.5, 1.0, math.nan, 2.0])
    got, lp = run(x, F32, u)
    assert got.tolist() == [0, 1, 2, 3, 3, 0, 3, 0, 3]
    assert np.allclose(lp, -math.log(4.0))
    got, _ = run(x, F32, u, k=[2] * 9)
    assert got.tolist() == [0, 0, 1, 1, 1, 0, 1, 0, 1]
    got, _ = run(x, F32, u, p=[0.5] * 9)
    assert got.tolist() == [0, 0, 1, 1, 1, 0, 1, 0, 1]


def test_draw_without_logp_repeats_and_frequencies():
    """The same call gives the same bits; uniforms k / 4096 draw every id as often as its probability says."""
    V, n = 300, 4096
    x = logits(1, V, F32, 14, std=1.0).expand(n, V).contiguous()
    u = torch.arange(n).float() / n
    a, lp = run(x, F32, u, T=[0.8] * n, k=[100] * n, p=[0.9] * n)
    c, _ = run(x, F32, u, T=[0.8] * n, k=[100] * n, p=[0.9] * n, logp=False)
    d, lp2 = run(x, F32, u, T=[0.8] * n, k=[100] * n, p=[0.9] * n)
    assert (a == c).all() and (a == d).all() and (lp == lp2).all()
    ids, w, _ = ref.kept_ids(x[0].double().cpu().numpy(), float(np.float32(0.8)), 100, float(np.float32(0.9)))
    count = np.bincount(a, minlength=V)
    assert count.sum() == n and set(np.flatnonzero(count)) <= set(ids)
    assert np.all(np.abs(count[ids] - n * w / w.sum()) <= 1.0 + 1e-6)  # an interval holds its length in grid points, +-1


def test_draw_beyond_32_bit_offsets():
    """Rows more than 2^32 elements apart in all (bf16, 8.7 GB of address range)."""
    V, stride = 5000, (1 << 31) + 24
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (3, V), (stride, 1))
    x.copy_(logits(3, V, BF16, 15))
    u = uniforms(3, 15)
    a = dict(T=[0.9] * 3, k=[0, 30, 0], p=[1.0, 0.9, 0.95])
    got, lp = run(x, BF16, u, **a)
    check(x, u, got, lp, **a)


def test_draw_on_streams_and_in_graphs():
    """Two calls at once on two streams, and a captured call replayed on new inputs."""
    V, n = 30011, 40
    x1, x2 = logits(n, V, F32, 16), logits(n, V, BF16, 17)
    u = uniforms(n, 16)
    T, p = [0.8] * n, [0.9] * n
    want1, _ = run(x1, F32, u, T=T, p=p)
    want2, _ = run(x2, BF16, u, T=T, p=p)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    dT, dp, du = dev(T, torch.float32), dev(p, torch.float32), u.to(DEV)
    t1, t2 = (torch.empty(n, dtype=torch.int32, device=DEV) for _ in range(2))
    torch.cuda.synchronize()
    for _ in range(5):
        assert b.domino_sample_filtered(x1, F32, x1.stride(0), dT, None, dp, None, du, n, V, t1, None, s1) == 0
        assert b.domino_sample_filtered(x2, BF16, x2.stride(0), dT, None, dp, None, du, n, V, t2, None, s2) == 0
    torch.cuda.synchronize()
    assert (t1.cpu().numpy() == want1).all() and (t2.cpu().numpy() == want2).all()
    x = x1.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rc = b.domino_sample_filtered(x, F32, x.stride(0), dT, None, dp, None, du, n, V, t1, None,
                                      torch.cuda.current_stream())
    assert rc == 0
    x.copy_(logits(n, V, F32, 18))
    du.copy_(uniforms(n, 19))
    graph.replay()
    torch.cuda.synchronize()
    check(x, du.cpu(), t1.cpu().numpy(), None, T=T, p=p)


def test_host_logits_pointer_of_another_kind_is_not_refused():
    """The device check looks at device memory alone: managed by the caller, pinned host memory is readable."""
    x = torch.randn((2, 500), generator=torch.Generator().manual_seed(20)).pin_memory()
    u = uniforms(2, 20).to(DEV)
    out = torch.empty(2, dtype=torch.int32, device=DEV)
    assert b.domino_sample_filtered(x, F32, 500, None, None, None, None, u, 2, 500, out, None,
                                    torch.cuda.current_stream()) == 0
    torch.cuda.synchronize()
    check(x, u.cpu(), out.cpu().numpy(), None)
