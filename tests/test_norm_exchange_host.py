"""The exchange of a row's sums between the warps that share it (norm_grad_kernel in csrc/norm.cu), as a model that goes through every order of
the warps' steps, on the CPU: a race of this kind shows on a GPU once in very many rows, if ever.

A warp sends the sums of row 0, then for each row i: it sends those of row i + 1, waits until all warps' sums of row i have arrived, reads
them, and (rows of one CTA only) meets the others at a barrier. Row i's sums lie in place i mod `places`. Whoever sends into a place in
which sums lie that some warp has not read yet, replaces them; a send takes effect at once here, which is the earliest that it can."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def overwrites(warps, rows, places, barrier):
    """The first (warp, row) in some order of steps whose sums replace unread ones; None if there is none."""
    steps = [("send", 0)]
    for i in range(rows):
        steps += [("send", i + 1)] * (i + 1 < rows) + [("read", i)] + [("arrive", i), ("leave", i)] * barrier
    position = {s: k for k, s in enumerate(steps)}
    done = lambda state, step: all(p > position[step] for p in state)
    start = (0,) * warps
    seen, todo = {start}, [start]
    while todo:
        state = todo.pop()
        for w in range(warps):
            if state[w] == len(steps):
                continue
            what, row = steps[state[w]]
            if what == "read" and not done(state, ("send", row)) or what == "leave" and not done(state, ("arrive", row)):
                continue
            if what == "send" and row >= places and not done(state, ("read", row - places)):
                return w, row
            following = state[:w] + (state[w] + 1,) + state[w + 1:]
            if following not in seen:
                seen.add(following)
                todo.append(following)
    assert (len(steps),) * warps in seen   # (and no order waits for good)
    return None


def places():
    with open(os.path.join(ROOT, "paper_2202_00774_b200", "csrc", "norm.cu")) as f:
        found = re.search(r"PLACES = CL > 1 \? (\d+) : (\d+);", f.read())
    return int(found.group(1)), int(found.group(2))


@pytest.mark.parametrize("warps", [2, 3])
def test_no_order_of_steps_replaces_sums_that_are_not_read(warps):
    cluster, cta = places()
    assert overwrites(warps, 8, cluster, False) is None
    assert overwrites(warps, 8, cta, True) is None


def test_the_model_finds_the_race_of_fewer_places():
    assert overwrites(2, 8, 3, False) is not None and overwrites(2, 8, 1, True) is not None
