"""The ring of stages of the gradients' tensor-core kernel (``csrc/grouped_gradient_tc.cu``) in every order in which its warps may run, on the CPU.

A barrier is the number of its completed phases, of which a wait sees the parity alone.  Three warps go by the ring: one fills a stage when the stage is empty, one multiplies,
and one looks at every stage and clears rows of some, for which the second waits."""
import os
import re

import pytest

from paper_2202_05008_b200 import build as B


def arrivals_in_the_source():
    with open(os.path.join(B.CSRC, "grouped_gradient_tc.cu")) as f:
        text = f.read()
    count = re.search(r"constexpr uint32_t kEmptyArrivals = (\d+);", text)
    assert "mbar_init(smem_u32(&empty[s]), kEmptyArrivals)" in text
    looks = text[text.index("} else if (warp == 10) {"):]
    looks = looks[:looks.index("} else {")]
    by_the_clearing_warp = len(re.findall(r"if \(lane == 0\) mbar_arrive\(smem_u32\(&empty\[stage\]\)\);", looks))
    return int(count.group(1)) if count else 1, by_the_clearing_warp


def outcomes(stages, clear, arrivals, clearer_arrives):
    """What can go wrong, over every interleaving: 'stuck', 'overtaken' (a warp finds another step in its stage), 'not cleared'."""
    steps = len(clear)
    passed = lambda completed, parity: (completed - 1) & 1 == parity        # a wait for the phase of that parity
    # (producer's, multiplier's and clearer's next step; completed phases of full and cleared; (phases, arrivals) of empty; what lies in each stage and whether it was cleared)
    start = (0, 0, 0, (0,) * stages, (0,) * stages, ((0, 0),) * stages, ((-1, False),) * stages, (0,) * stages)
    seen, todo, wrong = {start}, [start], set()

    def put(t, i, v):
        return t[:i] + (v,) + t[i + 1:]

    def arrive(empty, s):
        phases, n = empty[s]
        return put(empty, s, (phases + 1, 0) if n + 1 == arrivals else (phases, n + 1))
    while todo:
        state = todo.pop()
        p, m, c, full, cleared, empty, holds, turn_cleared = state
        moves = []
        if p < steps:
            s, parity = p % stages, p // stages & 1
            if passed(empty[s][0], parity ^ 1):
                moves.append((p + 1, m, c, put(full, s, full[s] + 1), cleared, empty, put(holds, s, (p, False)), turn_cleared))
        if m < steps:
            s, parity = m % stages, m // stages & 1
            if passed(cleared[s], turn_cleared[s]) if clear[m] else passed(full[s], parity):
                if holds[s][0] != m:
                    wrong.add("overtaken")
                elif clear[m] and not holds[s][1]:
                    wrong.add("not cleared")
                moves.append((p, m + 1, c, full, cleared, arrive(empty, s), holds, put(turn_cleared, s, turn_cleared[s] ^ 1) if clear[m] else turn_cleared))
        if c < steps:
            s, parity = c % stages, c // stages & 1
            if passed(full[s], parity):
                if holds[s][0] != c:
                    wrong.add("overtaken")
                after = put(holds, s, (holds[s][0], True)) if clear[c] else holds
                moves.append((p, m, c + 1, full, put(cleared, s, cleared[s] + 1) if clear[c] else cleared, arrive(empty, s) if clearer_arrives else empty, after, turn_cleared))
        if not moves and (p, m, c) != (steps,) * 3:
            wrong.add("stuck")
        for state in moves:
            if state not in seen:
                seen.add(state)
                todo.append(state)
    return wrong


def lists_of(steps):
    return [[bool(bits >> k & 1) for k in range(steps)] for bits in range(1 << steps)]


@pytest.mark.parametrize("stages,steps", [(2, 7), (3, 8), (4, 9)])
def test_no_order_of_the_warps_loses_a_phase(stages, steps):
    arrivals, by_the_clearing_warp = arrivals_in_the_source()
    assert by_the_clearing_warp == arrivals - 1
    for clear in lists_of(steps):
        assert not outcomes(stages, clear, arrivals, by_the_clearing_warp == 1), (stages, clear)


def test_a_ring_that_does_not_wait_for_the_clearing_warp_does():
    for stages in (2, 3, 4):
        clear = [False] * (2 * stages + 1)
        assert "stuck" in outcomes(stages, clear, 1, False)
        clear[-1] = True
        assert "stuck" in outcomes(stages, clear, 1, False)
        assert not outcomes(stages, [True] * (2 * stages + 1), 1, False)        # (where every step waits for it, it holds the ring)
