"""Attention over a paged cache whose copy of keys never lands: the waits run out (a second or two), the call ends with an
error status, and the next one on the same workspace is as ever.  Nothing traps, faults or hangs."""
import time

import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import paged_reference as ref
from tests.test_gpu_paged_attend import randq

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _call(p, q, ws, out, lse):
    assert b.domino_attend_paged(q, q.stride(0), q.shape[0], q.shape[1], p.cache, p.batch, p.D ** -0.5, b.DOMINO_MASK_CAUSAL, None, 0,
                                 out, out.stride(0), lse, ws, ws.numel(), torch.cuda.current_stream()) == 0
    return b.domino_check_status(ws, torch.cuda.current_stream())


# one tile of queries and two; the CTA takes a few tiles or many, near the beginning of the line, inside it and at its end
# (152 SMs: the stretches are 3, 14, 6 and 26 units, of which a group's first 12 hold no keys)
@pytest.mark.parametrize("kv,new,hq,hkv,cta", [([3000, 700], [1, 1], 8, 2, 6), ([6000, 9000], [1, 5], 8, 8, 100),
                                               ([3000, 500], [300, 33], 8, 2, 3), ([20000], [40], 32, 8, 148)])
def test_withheld_keys_time_out_then_the_next_call_is_right(kv, new, hq, hkv, cta):
    p = ref.Paged(kv, new, hkv, 128, b.DOMINO_BF16, 16, seed=cta)
    q = randq(p.tokens, hq, 128, b.DOMINO_BF16, 1)
    ws = torch.empty(b.domino_attend_workspace_bytes(p.tokens, hq, p.cache), dtype=torch.uint8, device=DEV)
    want, want_lse = torch.empty_like(q), torch.empty((p.tokens, hq), device=DEV)
    assert _call(p, q, ws, want, want_lse) == 0
    out, lse = torch.empty_like(q), torch.empty_like(want_lse)
    assert b.domino_debug_hold(b.DOMINO_HOLD_KEY_TILE, cta) == 0
    t0 = time.perf_counter()
    try:
        status = _call(p, q, ws, out, lse)
    finally:
        assert b.domino_debug_hold(b.DOMINO_HOLD_OFF) == 0
    assert status == b.DOMINO_ERR_TIMEOUT, b.domino_status_string(status)
    assert 0.5 < time.perf_counter() - t0 < 30.0
    # rows that the CTA had no part in are as without the hook
    assert bool((lse == want_lse).any())
    for _ in range(2):  # the hook held one launch only
        out.zero_()
        assert _call(p, q, ws, out, lse) == 0
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_a_cta_that_the_launch_has_not_withholds_nothing():
    p = ref.Paged([100], [1], 2, 64, b.DOMINO_BF16, 16, seed=1)
    q = randq(1, 4, 64, b.DOMINO_BF16, 1)
    ws = torch.empty(b.domino_attend_workspace_bytes(1, 4, p.cache), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(q), torch.empty((1, 4), device=DEV)
    assert b.domino_debug_hold(b.DOMINO_HOLD_KEY_TILE, 1 << 20) == 0
    assert _call(p, q, ws, out, lse) == 0
