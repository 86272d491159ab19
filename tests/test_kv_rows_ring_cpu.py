"""The ring of stages of the attention of many rows, without a GPU: its roles as steps over barriers with phases, taken in any order.
What a barrier waits for is read from the kernel's source, so that the model and the kernel do not part ways."""
import os
import random
import re

import pytest

import paper_2606_17059_gb300 as g

SOURCE = open(os.path.join(g._build.CSRC, "kv_rows.cuh")).read()
HELPERS = SOURCE[SOURCE.index("infinities and NaN among values that not all rows see"):]
EMPTY = int(re.search(r"bar_init\(sh\.empty\[i\], (\d+)\)", SOURCE).group(1))      # arrivals that free a stage
HELPERS_FREE = "bar_arrive(sh.empty[stage])" in HELPERS                            # whether the helpers are among them
BOXES = int(re.search(r"bar_init\(sh\.q_raw\[i\], a\.boxes \? (\d+) : 64\)", SOURCE).group(1))  # arrivals with queries that one helper brings by boxes
BOTH = "if (mine == 32) bar_arrive(there);" in HELPERS                             # whether the other one is among them


class Barrier:
    """Phases that complete with `count` arrivals; a wait for a parity passes once the phase under way has the other one."""

    def __init__(self, count):
        self.count, self.left, self.phase = count, count, 0

    def arrive(self):
        self.left -= 1
        assert self.left >= 0
        if self.left == 0:
            self.left, self.phase = self.count, self.phase + 1

    def passed(self, parity):
        return (self.phase & 1) != parity


def run(roles, rng, slow):
    """Takes steps of the roles (generators that yield what they wait for) in random order; `slow`: of these seldom."""
    waits = {name: (lambda: True) for name in roles}
    while roles:
        names = [n for n in roles if waits[n]()]
        assert names, "nobody can go on: " + ", ".join(roles)
        ready = [n for n in names if n not in slow or rng.random() < 0.02] or names
        n = rng.choice(ready)
        try:
            waits[n] = next(roles[n])
        except StopIteration:
            del roles[n]


@pytest.mark.parametrize("stages", [3, 4, 6, 8])
@pytest.mark.parametrize("slow", [(), ("helper 0",), ("helper 0", "helper 1"), ("products",), ("copies",)])
def test_no_role_falls_a_turn_behind(stages, slow):
    for seed in range(40):
        rng = random.Random(seed)
        total = 60
        looked_at = [rng.random() < 0.2 for _ in range(total)]    # values that not all rows see
        full, empty, checked = ([Barrier(n) for _ in range(stages)] for n in (1, EMPTY, 2))
        held = [-1] * stages
        done = [set() for _ in range(total)]

        def copies():
            for t in range(total):
                s, phase = t % stages, t // stages & 1
                yield lambda: empty[s].passed(phase ^ 1)
                held[s] = t
                full[s].arrive()

        def products():
            for t in range(total):
                s, phase = t % stages, t // stages & 1
                yield lambda: full[s].passed(phase)
                if looked_at[t]:
                    yield lambda: checked[s].passed(phase)
                    assert len(done[t]) == 2, "values that were not looked at"
                assert held[s] == t
                empty[s].arrive()

        def helper(me):
            for t in range(total):
                s, phase = t % stages, t // stages & 1
                yield lambda: full[s].passed(phase)
                assert held[s] == t, "a stage that holds something else by now"
                done[t].add(me)
                checked[s].arrive()
                if HELPERS_FREE:
                    empty[s].arrive()

        run({"copies": copies(), "products": products(), "helper 0": helper(0), "helper 1": helper(1)}, rng, slow)


@pytest.mark.parametrize("boxes", [False, True])
@pytest.mark.parametrize("slow", [(), ("helper 0",), ("helper 1",), ("products",)])
def test_queries_come_and_go(boxes, slow):
    for seed in range(40):
        rng = random.Random(seed)
        units = 30
        there, free = Barrier(BOXES if boxes else 2), Barrier(1)
        brought = [set() for _ in range(units)]

        def helper(me):
            for u in range(units):
                yield lambda: free.passed((u & 1) ^ 1)
                assert u == 0 or free.phase == u, "a phase that is another's"
                brought[u].add(me)
                if not boxes or me == 0 or BOTH:
                    there.arrive()

        def products():
            for u in range(units):
                yield lambda: there.passed(u & 1)
                assert 0 in brought[u]
                free.arrive()

        run({"products": products(), "helper 0": helper(0), "helper 1": helper(1)}, rng, slow)
