"""The hook that withholds keys: its constant is the header's, negative CTAs are refused before any device call (CPU)."""
import os
import re

from paper_2605_29707_gb300 import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_constant_and_refusal():
    with open(os.path.join(ROOT, "include", "domino.h")) as f:
        m = re.search(r"DOMINO_HOLD_KEY_TILE = (\d+)", f.read())
    assert int(m.group(1)) == b.DOMINO_HOLD_KEY_TILE
    assert b.domino_debug_hold(b.DOMINO_HOLD_KEY_TILE, -1) == b.DOMINO_ERR_INVALID_ARG
