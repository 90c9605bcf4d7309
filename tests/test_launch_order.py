"""Programmatic dependent launches: a kernel releases its successor only behind its own wait for its predecessor.

Kernels that may fetch weights before their wait (MATQ_GEMV_PDL) rely on that: only then is the direct predecessor the one kernel that can still be
running.  Which kernel runs when cannot be forced from a test, so the sources are read."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06786_b200", "csrc")
WAIT = r'(?:after_previous_kernel\(\);|asm volatile\("griddepcontrol\.wait;" ::: "memory"\);)'
RELEASE = r'(?:let_next_kernel_start\(\);|asm volatile\("griddepcontrol\.launch_dependents;"\);)'
# Kernels that start behind a kernel of the same call which itself waited before it released them, and which writes nothing that a later kernel reads early.
BEHIND_THEIR_OWN_CALL = {"slice_pack_ep": r"^\s{4}let_next_kernel_start\(\);", "gemv_stream": r"if \(P\.pdl == 2\) asm volatile"}
FILES = sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh")))


def _kernels(text):
    """(name, body) of every __global__ function."""
    for m in re.finditer(r"__global__", text):
        opening = text.index("{", m.start())
        name = re.findall(r"(\w+)\s*\(", text[m.start():opening])
        name = [n for n in name if n not in ("__launch_bounds__", "__cluster_dims__", "__align__")][0]
        depth, at = 0, opening
        while True:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
            if depth == 0:
                break
        yield name, text[opening:at]


@pytest.mark.parametrize("name", FILES)
def test_release_follows_the_wait(name):
    text = re.sub(r"//[^\n]*|[^\n]*void let_next_kernel_start[^\n]*", "", open(os.path.join(CSRC, name)).read())
    inside = 0
    for kernel, body in _kernels(text):
        first_wait = re.search(r"^ {4}" + WAIT, body, flags=re.M)                # not under a condition
        for m in re.finditer(RELEASE, body):
            inside += 1
            line = body[body.rfind("\n", 0, m.start()) + 1:m.end()]
            ok = (re.search(WAIT + r"\s*$", body[:m.start()]) or (first_wait and first_wait.start() < m.start())
                  or (kernel in BEHIND_THEIR_OWN_CALL and re.search(BEHIND_THEIR_OWN_CALL[kernel], line)))
            assert ok, f"{name}: {kernel} releases its successor before its own wait: {line.strip()}"
    total = len(re.findall(RELEASE, text))
    assert inside == total, f"{name}: a release outside a kernel's body is not covered by this test"


def test_some_kernels_are_checked():
    assert sum(len(re.findall(RELEASE, open(os.path.join(CSRC, f)).read())) for f in FILES) >= 15
