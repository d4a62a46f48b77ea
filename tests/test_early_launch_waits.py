"""Kernels that may start before the kernel ahead of them has ended wait for it before they touch
memory: griddepcontrol.wait makes the earlier kernels' results visible to the grid that executes it,
and to no grid that this one lets start."""
import os
import re

import pytest

from test_early_launch_loads import FILES, closing, code_of, kernels

WAIT = re.compile(r"griddepcontrol\.wait|\bpdl_wait\(\)")
#: Global memory: TMA loads and stores, subscripts and member calls of a struct's pointers (p.x[..]),
#: and what the window kernels read through (sequence lengths, tiles made of them).
TOUCHES = re.compile(r"\b(tma_\w+|load_box|store_box|load_tile|load_rows|load_raw|seq_len|atomic\w+)\s*[(<]|"
                     r"\b(KeyWork|QueryTile) \w+\(|\bp\.\w+(\.\w+)?\[")


def helpers(path):
    """Bodies of the device functions of a file, by name."""
    text = code_of(path)
    found = {}
    for m in re.finditer(r"__device__\s+__forceinline__\s+[\w:]+\s+(\w+)\s*(?=\()", text):
        end = closing(text, m.end(), "()")
        if text[end:].lstrip().startswith("{"):
            body = text.index("{", end)
            found[m.group(1)] = text[body:closing(text, body, "{}")]
    return found


def early(body, wait):
    """What a body touches before the wait at ``wait`` (lambdas that are only defined there count too)."""
    return [m.group(0) for m in TOUCHES.finditer(body[:wait])]


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_the_wait_comes_before_memory_is_touched(path):
    inner = helpers(path)
    for name, _, body in kernels(path):
        at = WAIT.search(body)
        if at is not None:
            assert early(body, at.start()) == [], name
            continue
        # a kernel whose first step, in a function of its own, is the wait
        calls = [(m.start(), f) for f in inner if WAIT.search(inner[f])
                 for m in [re.search(r"\b" + f + r"\s*[(<]", body)] if m]
        if calls:
            start, f = min(calls)
            assert early(body, start) == [] and early(inner[f], WAIT.search(inner[f]).start()) == [], name


def test_window_kernels_wait_themselves():
    """Each of them starts early (they are all launched that way), so each has a wait of its own."""
    for path in FILES:
        if not os.path.basename(path).startswith(("window_", "qk_norm")):
            continue
        inner = helpers(path)
        for name, _, body in kernels(path):
            assert WAIT.search(body) or any(re.search(r"\b" + f + r"\s*[(<]", body)
                                            for f in inner if WAIT.search(inner[f])), name


def test_a_wait_at_the_end_is_found():
    """Mistakes planted in a kernel's text."""
    good = "{ init(); pdl_wait(); x = p.lse[3]; load_box(a); }"
    assert early(good, WAIT.search(good).start()) == []
    for bad in ("{ x = p.lse[3]; pdl_wait(); }", "{ load_box(a, p.q); pdl_wait(); }",
                "{ const KeyWork w(p, 0); pdl_wait(); }"):
        assert early(bad, WAIT.search(bad).start()), bad
