"""No kernel touches another CTA's shared memory before a cluster barrier has shown that the CTA runs (read from the text
of csrc/, no GPU): a remote access to a CTA that has not started is undefined, and which CTA starts last is not ours to
say, so no run can show that it is missing."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_29707_gb300", "csrc")
REMOTE = re.compile(r"(?:\b(?:ld|st|atom|red)\b|mbarrier\.arrive)[\w.]*shared::cluster")
HEAD = re.compile(r"(__global__|__device__)[^;{}]*?\b(\w+)\s*\([^;{}]*\)\s*(?:const\s*)?\{")
CALL = re.compile(r"\b(\w+)\s*(?:<[^;(){}]*>)?\(|" + REMOTE.pattern)


def _code():
    text = ""
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".cu", ".cuh")):
            with open(os.path.join(CSRC, name)) as f:
                text += re.sub(r"//[^\n]*", "", f.read()) + "\n"
    return text


def _functions(text):
    """({kernel: body}, {device function: body}); overloads' bodies one after another."""
    kernels, functions = {}, {}
    for m in HEAD.finditer(re.sub(r"__launch_bounds__\([^)]*\)", lambda m: " " * len(m.group()), text)):
        depth, at = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        into = kernels if m.group(1) == "__global__" else functions
        into[m.group(2)] = into.get(m.group(2), "") + text[m.end():at]
    return kernels, functions


def _events(body, functions, inside=()):
    """'A' arrive, 'W' wait, 'R' remote access, in the order of the text, called functions at their calls."""
    out = ""
    for m in CALL.finditer(body):
        name = m.group(1)
        if name is None:
            out += "R"
        elif name == "cluster_sync":
            out += "AW"
        elif name in ("cluster_arrive", "cluster_wait"):
            out += "A" if name == "cluster_arrive" else "W"
        elif name in functions and name not in inside:
            out += _events(functions[name], functions, inside + (name,))
    return out


KERNELS, FUNCTIONS = _functions(_code())
WITH_REMOTE = sorted(k for k, body in KERNELS.items() if "R" in _events(body, FUNCTIONS))


def test_the_kernels_with_remote_accesses_are_found():
    assert {"distill_kernel", "filtered_draw_kernel"} <= set(WITH_REMOTE)


@pytest.mark.parametrize("kernel", WITH_REMOTE)
def test_a_cluster_barrier_precedes_the_first_remote_access(kernel):
    events = _events(KERNELS[kernel], FUNCTIONS)
    before = events[:events.index("R")]
    assert "W" in before and before.index("A") < before.index("W"), events
