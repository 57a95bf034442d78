"""Argument errors of the entry points on a paged cache come back before anything is enqueued, and the binding's
structures have the header's layout (CPU)."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2605_29707_gb300 import binding as b

BAD, UNSUP = b.DOMINO_ERR_INVALID_ARG, b.DOMINO_ERR_UNSUPPORTED
P = 1 << 12  # an aligned non-null stand-in; never dereferenced because validation fails first
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CACHE = dict(k=P, v=2 * P, page_stride=16 * 2 * 64, token_stride=2 * 64, head_stride=64, pages=8, page=16, heads=2, head_dim=64,
             dtype=b.DOMINO_BF16)
BATCH = dict(table=P, table_stride=4, table_width=4, kv_len=P, start=P, B=3)

CACHE_FAULTS = [(dict(k=None), BAD), (dict(v=None), BAD), (dict(k=P + 1), BAD), (dict(pages=0), BAD), (dict(page=0), BAD),
                (dict(heads=0), BAD), (dict(head_dim=0), BAD), (dict(head_dim=257), UNSUP), (dict(dtype=3), UNSUP),
                (dict(dtype=-1), UNSUP), (dict(page_stride=63), BAD), (dict(token_stride=-64), BAD), (dict(head_stride=0), BAD),
                (dict(page_stride=1 << 62), BAD), (dict(heads=1 << 15), UNSUP)]
BATCH_FAULTS = [(dict(table=None), BAD), (dict(table=P + 2), BAD), (dict(kv_len=None), BAD), (dict(start=None), BAD),
                (dict(start=P + 1), BAD), (dict(B=0), BAD), (dict(table_width=0), BAD), (dict(table_stride=3), BAD)]


def _shared(kw):
    cache, batch = dict(CACHE), dict(BATCH)
    for name in list(kw):
        if name in cache and name not in ("k", "v") or name in ("cache_k", "cache_v"):
            cache[name.replace("cache_", "")] = kw.pop(name)
        elif name in batch:
            batch[name] = kw.pop(name)
    return b.make_cache(**cache), b.make_batch(**batch)


def _append(**kw):
    c, t = _shared(kw)
    a = dict(q=P, q_stride=256, k=P, k_stride=128, v=P, v_stride=128, positions=None, tree_depth=P, N=4, freq=P, amplitude=1.0,
             layout=b.DOMINO_ROPE_HALF, rot=64, q_heads=4, tokens=5, q_out=2 * P, q_out_stride=256, cache=c, batch=t)
    a.update(kw)
    return b.domino_rope_append(**a)


def _attend(**kw):
    c, t = _shared(kw)
    a = dict(q=P, q_stride=256, tokens=5, q_heads=4, cache=c, batch=t, scale=0.125, mask=b.DOMINO_MASK_TREE, tree_parent=P, N=4,
             out=2 * P, out_stride=256, lse=P, workspace=P, workspace_bytes=1 << 30)
    a.update(kw)
    return b.domino_attend_paged(**a)


def _commit(**kw):
    c, t = _shared(kw)
    a = dict(cache=c, batch=t, layers=2, layer_stride=1 << 20, accepted_nodes=P, accepted_count=P, N=4, new_len=2 * P)
    a.update(kw)
    return b.domino_cache_commit(**a)


def _rope(**kw):
    a = dict(x=P, dtype=b.DOMINO_BF16, x_token_stride=256, x_head_stride=64, positions=P, freq=P, amplitude=1.0,
             layout=b.DOMINO_ROPE_PAIRS, gradient=0, tokens=5, heads=4, head_dim=64, rot=64, y=2 * P, y_token_stride=256,
             y_head_stride=64)
    a.update(kw)
    return b.domino_rope(**a)


@pytest.mark.parametrize("call", [_append, _attend, _commit])
@pytest.mark.parametrize("kw,code", [({("cache_" + n if n in ("k", "v") else n): x for n, x in kw.items()}, code)
                                     for kw, code in CACHE_FAULTS] + BATCH_FAULTS + [(dict(cache=None), BAD), (dict(batch=None), BAD)])
def test_cache_and_batch_refusals(call, kw, code):
    kw = dict(kw)
    if call is _attend and kw.get("heads") == 1 << 15:
        kw["q_heads"] = 1 << 15
    assert call(**kw) == code


ROTATION = [(dict(rot=-2), BAD), (dict(rot=63), BAD), (dict(rot=66), BAD), (dict(freq=None), BAD), (dict(freq=P + 2), BAD),
            (dict(amplitude=float("nan")), BAD), (dict(amplitude=float("inf")), BAD), (dict(layout=2), BAD), (dict(layout=-1), BAD),
            (dict(tokens=0), BAD)]


@pytest.mark.parametrize("kw,code", ROTATION + [
    (dict(x=None), BAD), (dict(y=None), BAD), (dict(positions=None), BAD), (dict(positions=P + 2), BAD), (dict(x=P + 1), BAD),
    (dict(y=2 * P + 1), BAD), (dict(dtype=3), UNSUP), (dict(heads=0), BAD), (dict(head_dim=0), BAD), (dict(head_dim=257), UNSUP),
    (dict(x_token_stride=63), BAD), (dict(y_head_stride=-64), BAD), (dict(x_token_stride=1 << 62), BAD),
    (dict(y=P, y_token_stride=512), BAD), (dict(y=P, y_head_stride=128), BAD)])
def test_rope_refusals(kw, code):
    assert _rope(**kw) == code


@pytest.mark.parametrize("kw,code", ROTATION + [
    (dict(q=None), BAD), (dict(k=None), BAD), (dict(v=None), BAD), (dict(q_out=None), BAD), (dict(q=P + 1), BAD), (dict(k=P + 1), BAD),
    (dict(q_heads=-1), BAD), (dict(q_stride=255), BAD), (dict(k_stride=127), BAD), (dict(v_stride=127), BAD),
    (dict(q_out_stride=255), BAD), (dict(q_out=P, q_out_stride=512), BAD), (dict(positions=P), BAD), (dict(N=-1), BAD),
    (dict(tree_depth=P + 2), BAD), (dict(q_heads=1 << 15, q_stride=1 << 22), UNSUP)])
def test_rope_append_refusals(kw, code):
    assert _append(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=0), BAD), (dict(q_heads=0), BAD), (dict(q_heads=3), BAD), (dict(q_heads=2 * 129), UNSUP), (dict(q=None), BAD),
    (dict(out=None), BAD), (dict(q=P + 1), BAD), (dict(out=P + 1), BAD), (dict(q_stride=255), BAD), (dict(out_stride=255), BAD),
    (dict(out=P, out_stride=512), BAD), (dict(mask=3), BAD), (dict(mask=-1), BAD), (dict(tree_parent=None), BAD),
    (dict(tree_parent=P + 2), BAD), (dict(N=-1), BAD), (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD),
    (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD), (dict(scale=1e-39), BAD), (dict(scale=3e38), BAD),
    (dict(lse=P + 2), BAD), (dict(workspace=None), BAD), (dict(workspace=P + 128), BAD)])
def test_attend_refusals(kw, code):
    assert _attend(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(layers=0), BAD), (dict(layers=1 << 15), UNSUP), (dict(layer_stride=63), BAD), (dict(N=-1), BAD), (dict(N=(1 << 20) + 1), BAD),
    (dict(accepted_nodes=None), BAD), (dict(accepted_count=None), BAD), (dict(new_len=None), BAD), (dict(new_len=P), BAD), (dict(accepted_count=2 * P), BAD),
    (dict(accepted_nodes=P + 2), BAD), (dict(accepted_count=P + 2), BAD), (dict(new_len=2 * P + 2), BAD)])
def test_commit_refusals(kw, code):
    assert _commit(**kw) == code


def test_workspace_of_refused_sizes_is_nothing():
    c = b.make_cache(**CACHE)
    assert b.domino_attend_workspace_bytes(0, 4, c) == 0
    assert b.domino_attend_workspace_bytes(5, 3, c) == 0
    assert b.domino_attend_workspace_bytes(5, 4, None) == 0


def test_status_string_of_a_bad_page():
    assert b.domino_status_string(b.DOMINO_ERR_BAD_PAGE) == "DOMINO_ERR_BAD_PAGE"


@pytest.mark.parametrize("struct", [b.domino_kv_cache, b.domino_kv_batch])
def test_structures_match_the_header(struct, tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    name, fields = struct.__name__, [f for f, _ in struct._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(
        ["#include <stddef.h>", "#include <stdio.h>", '#include "domino.h"', "int main(void) {",
         f'  printf("sizeof %zu\\n", sizeof({name}));'] +
        [f'  printf("{f} %zu\\n", offsetof({name}, {f}));' for f in fields] + ["  return 0;", "}"]))
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True, capture_output=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    c = {n: int(x) for n, x in (line.split() for line in out.splitlines())}
    assert c["sizeof"] == ctypes.sizeof(struct)
    assert all(c[f] == getattr(struct, f).offset for f in fields)
