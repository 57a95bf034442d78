"""Tree verification under temperature, top-k, top-p and min-p (domino_verify_tree_filtered): the draws against
the plain 64-bit form (bounds in test_gpu_sample_filtered.py), the walk against the oracle's on those draws."""
import numpy as np
import pytest
import torch

import oracle
from paper_2605_29707_gb300 import binding as b, inputs
from tests import rows_reference as ref
from tests.test_gpu_sample_filtered import BORDER, DEV, TYPES, dev

pytestmark = pytest.mark.gpu


def _run(case, dtype, u, T, k, p, m, pad=0):
    B, N = case.parent.shape
    V = case.target.shape[2]
    rows = B * (N + 1)
    x = torch.full((rows, V + pad), float("inf"), dtype=TYPES[dtype], device=DEV)
    x[:, :V] = torch.from_numpy(case.target).view(rows, V).to(DEV).to(TYPES[dtype])
    par, tok = torch.from_numpy(case.parent).to(DEV), torch.from_numpy(case.token).to(DEV)
    out = {n: torch.full(s, -7, dtype=torch.int32, device=DEV)
           for n, s in (("y", (B, N + 1)), ("nodes", (B, max(N, 1))), ("count", (B,)), ("bonus", (B,)))}
    lp = torch.empty((B, N + 1), device=DEV)
    keep = (dev(T, torch.float32), dev(k, torch.int32), dev(p, torch.float32), dev(m, torch.float32), u.to(DEV))
    rc = b.domino_verify_tree_filtered(x, dtype, V + pad, par if N else None, tok if N else None, *keep, B, N, V,
                                       out["y"], lp, out["nodes"] if N else None, out["count"], out["bonus"],
                                       torch.cuda.current_stream())
    assert rc == 0, b.domino_status_string(rc)
    torch.cuda.synchronize()
    return x[:, :V].double().cpu().numpy().reshape(B, N + 1, V), {n: t.cpu().numpy() for n, t in out.items()}, lp.cpu()


@pytest.mark.parametrize("B,N,V,dtype,pad,chain", [
    (3, 16, 1000, b.DOMINO_F32, 0, False), (2, 20, 999, b.DOMINO_BF16, 3, False), (5, 12, 257, b.DOMINO_F16, 0, True),
    (2, 40, 4096, b.DOMINO_BF16, 0, False), (1, 1, 5, b.DOMINO_F32, 0, False), (4, 0, 300, b.DOMINO_F32, 0, False),
    (2, 16, 151936, b.DOMINO_BF16, 0, False)])
def test_verify_filtered_matches_the_plain_form(B, N, V, dtype, pad, chain):
    c = inputs.make_verify_case(B, N, V, 60 + N, p_plant=0.9, chain=chain, margin=3.0)
    u = torch.rand((B, N + 1), generator=torch.Generator().manual_seed(V))
    T = [(0.7, 1.0, 1.3, 0.0, 0.5)[i % 5] for i in range(B)]
    k = [(50, 0, 3, 20, 1000)[i % 5] for i in range(B)]
    p = [(0.9, 0.8, 1.0, 0.95, 0.7)[i % 5] for i in range(B)]
    m = [(0.0, 0.05, 0.01, 0.0, 0.1)[i % 5] for i in range(B)]
    x, out, lp = _run(c, dtype, u, T, k, p, m, pad)
    accepted = 0
    for s in range(B):
        for r in range(N + 1):
            e, elp, margin = ref.draw(x[s, r], float(u[s, r]), float(np.float32(T[s])), k[s], float(np.float32(p[s])),
                                      float(np.float32(m[s])))
            assert margin < BORDER or out["y"][s, r] == e, (s, r)
            assert margin < BORDER or abs(float(lp[s, r]) - elp) <= 2.0 ** -21 * (1 + abs(elp) + np.log(V))
        nodes, bonus = oracle.tree_walk(c.parent[s], c.token[s], out["y"][s])
        assert int(out["count"][s]) == len(nodes) and int(out["bonus"][s]) == bonus
        if N:
            assert out["nodes"][s, :len(nodes)].tolist() == nodes.tolist() and (out["nodes"][s, len(nodes):N] == -1).all()
        accepted += len(nodes)
    assert accepted > 0 or N < 10


def test_verify_filtered_greedy_rows_are_the_greedy_verification():
    B, N, V = 3, 16, 4096
    c = inputs.make_verify_case(B, N, V, 71, p_plant=0.8)
    _, out, _ = _run(c, b.DOMINO_F32, torch.rand((B, N + 1)), [0.0] * B, None, None, None)
    ra, gn = torch.empty((B, N + 1), dtype=torch.int32, device=DEV), torch.empty((B, N), dtype=torch.int32, device=DEV)
    gc, gb = (torch.empty((B,), dtype=torch.int32, device=DEV) for _ in range(2))
    rc = b.domino_verify_tree_greedy(torch.from_numpy(c.target).to(DEV), torch.from_numpy(c.parent).to(DEV),
                                     torch.from_numpy(c.token).to(DEV), B, N, V, ra, gn, gc, gb,
                                     torch.cuda.current_stream())
    assert rc == 0
    torch.cuda.synchronize()
    for n, t in (("y", ra), ("nodes", gn), ("count", gc), ("bonus", gb)):
        np.testing.assert_array_equal(out[n], t.cpu().numpy())


def test_verify_filtered_in_a_graph():
    B, N, V = 4, 16, 5000
    c = inputs.make_verify_case(B, N, V, 72, p_plant=0.9, margin=4.0)
    u = torch.rand((B, N + 1), generator=torch.Generator().manual_seed(1))
    T, p = [0.8] * B, [0.9] * B
    _, want, _ = _run(c, b.DOMINO_F32, u, T, None, p, None)
    x, par, tok = (torch.from_numpy(a).to(DEV) for a in (c.target, c.parent, c.token))
    y, nodes = torch.empty((B, N + 1), dtype=torch.int32, device=DEV), torch.empty((B, N), dtype=torch.int32, device=DEV)
    count, bonus = (torch.empty((B,), dtype=torch.int32, device=DEV) for _ in range(2))
    dT, dp, du = dev(T, torch.float32), dev(p, torch.float32), u.to(DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rc = b.domino_verify_tree_filtered(x, b.DOMINO_F32, V, par, tok, dT, None, dp, None, du, B, N, V, y, None, nodes,
                                           count, bonus, torch.cuda.current_stream())
    assert rc == 0
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for n, t in (("y", y), ("nodes", nodes), ("count", count), ("bonus", bonus)):
        np.testing.assert_array_equal(want[n], t.cpu().numpy())
