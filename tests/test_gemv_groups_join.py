"""gemv_groups: the CTAs of a cluster add their sums over row steps, in two buffers that take turns, and meet a step late.

Which CTA runs ahead cannot be forced from a test, so the order of the kernel's accesses and barriers is read from its source, and every interleaving of two
CTAs that follow it is walked: no sums may be gathered from a buffer that holds those of another step."""
import os
import re

import pytest

from paper_2502_06786_b200 import binding as mq

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06786_b200", "csrc", "groups.cu")
EVENTS = {"write": r"part\[i\] = sum;", "wait": r"cluster_wait\(\);", "gather": r"gather\(before,", "arrive": r"cluster_arrive\(\);"}


def _events(text):
    return [name for _, name in sorted((m.start(), name) for name, e in EVENTS.items() for m in re.finditer(e, text))]


def _order():
    """Events of a row step, and of what follows the last one."""
    text = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    kernel = text[text.index("gemv_groups_kernel(const GemvParams P) {"):]
    at = kernel.index("for (int step = blockIdx.y;")
    at = kernel.index("{", at)
    depth, end = 0, at
    while True:
        depth += {"{": 1, "}": -1}.get(kernel[end], 0)
        end += 1
        if depth == 0:
            break
    return _events(kernel[at:end]), _events(kernel[end:kernel.index("struct GemvPlan")])


def _program(steps, order):
    step, last = order
    out = []
    for s in range(steps):
        for e in step:
            if e in ("wait", "gather") and s == 0:
                continue                                         # no step before
            out.append((e, s - 1 if e == "gather" else s))
    return out + [(e, steps - 1) for e in last]


def _stale(steps, order):
    """Whether some interleaving of two CTAs gathers the sums of another step."""
    program = _program(steps, order)
    start = ((0, 0), ((None, None), (None, None)), (0, 0))       # where each CTA is, what its buffers hold, its arrivals
    seen, todo = {start}, [start]
    ended = False
    while todo:
        at, held, arrived = todo.pop()
        ended |= at == (len(program), len(program))
        for me in (0, 1):
            if at[me] == len(program):
                continue
            e, s = program[at[me]]
            buffers, counts = [list(h) for h in held], list(arrived)
            if e == "wait" and counts[1 - me] < counts[me]:
                continue
            if e == "gather" and any(h[s % 2] != s for h in held):
                return True
            if e == "write":
                buffers[me][s % 2] = s
            if e == "arrive":
                counts[me] += 1
            state = (tuple(p + (i == me) for i, p in enumerate(at)), tuple(map(tuple, buffers)), tuple(counts))
            if state not in seen:
                seen.add(state)
                todo.append(state)
    assert ended                                                 # no interleaving is needed that never comes
    return False


def test_no_sums_of_another_step_are_gathered():
    order = _order()
    assert sorted(order[0]) == ["arrive", "gather", "wait", "write"] and order[1] == ["wait", "gather", "arrive", "wait"]
    for steps in range(1, 8):
        assert not _stale(steps, order), f"{steps} steps: {order[0]}"


def test_the_walk_finds_a_buffer_that_is_written_too_early():
    late = (["write", "wait", "gather", "arrive"], ["wait", "gather", "arrive", "wait"])
    assert not _stale(2, late) and _stale(3, late)


def test_plan_refusals_and_choices():
    plan = mq.gemv_groups_plan
    for M, N, K, group, st in ((0, 8, 256, 64, mq.ERR_INVALID_ARG), (2, 0, 256, 64, mq.ERR_INVALID_ARG), (2, -1, 256, 64, mq.ERR_INVALID_ARG), (2, 8, -64, 64, mq.ERR_INVALID_ARG),
                               (2, 8, 256, 16, mq.ERR_UNSUPPORTED), (2, 8, 250, 64, mq.ERR_SHAPE), (2, 8, 0, 64, mq.ERR_SHAPE), (2, 8, 65600, 32, mq.ERR_SHAPE),
                               (2, 1 << 31, 256, 64, mq.ERR_SHAPE), (1 << 40, 8, 256, 64, mq.ERR_SHAPE)):
        with pytest.raises(mq.MatqError) as e:
            plan(M, N, K, group)
        assert e.value.status == st, (M, N, K, group)
    assert mq._lib.matq_gemv_groups_plan(2, 8, 256, 64, None, None, None) == mq.OK
    tokens, parts, steps = plan(16, 28672, 8192, 128)
    assert tokens == 16 and parts > 1 and steps > 2
